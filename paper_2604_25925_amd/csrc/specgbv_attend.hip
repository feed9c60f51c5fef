// Attention of new queries over a paged cache, split over the cache's length and joined.
//
//   out = sum_j w_j v_j / sum_j w_j,   w_j = 2^(c <q, k_j> - m),   c = scale log2(e),
// in one pass over the keys with a running reference m per query (any m gives the same quotient; it is raised, and what has been
// summed is scaled, only where a weight would exceed 2^8, so that tiles after the first few seldom pay for it).  One operation gives
// c <q, k> - m; what the rounding of m leaves out is a factor of all weights, but a vast one where scores lie near the type's lowest
// value, so there (|m| > 2^20) the product is rounded before m is taken off.
//
// Rows.  A kv head's queries of one sequence (tokens x heads of its group), or of all drafts of a prefix while the keys lie in pages
// that the drafts share, are the rows of a matrix product: one read of a key serves them all.  A wave holds 16 RT rows.
//
// A tile is 32 keys (bfloat16; 16 in float32); where the waves of a workgroup share its rows it never leaves registers.  The product is formed as keys x rows: in the
// result a lane holds scores of ONE row (lane % 16) and, because the product's row m is made key 8 (m / 4) + 4 h + m % 4 of the tile (h: which
// half), of 8 ADJACENT keys, those of run lane / 16.  That is the layout in which the second product (values^T x weights) takes its
// right operand, so the weights go from one product to the next without leaving their lane, and a lane loads the values of its own run
// of keys: whole rows, each used entry by entry (two 16-bit halves put together by one byte permutation).  The order of entries within the
// contraction over head_dim is free, so lanes take 16-byte pieces of keys.
//
// WK = 0 (few rows, short): each wave by itself.  4 (few rows): the waves of a workgroup take the tiles in turn and join at the end through LDS; neither the keys nor the values pass
// through LDS, and no barrier stands in the loop.  1: each wave has rows of its own, and the
// waves share the tiles, which come into LDS by asynchronous loads two tiles ahead, and the values are read turned.  Straight into registers each 16-byte piece of a key is
// a line of its own for the cache (16 neighbouring lanes hold 16 rows), 750 accesses a tile, which bounded it with many rows; through LDS
// neighbouring lanes load neighbouring pieces, once for four waves.  In LDS piece n of key m lies in slot n ^ m, so that 8 lanes that read one
// piece of 8 keys meet 8 groups of banks.
//
// The split.  A unit (a sequence, or a prefix with its drafts) is cut into parts over its length, so that a launch fills the card once and all
// workgroups have the same number of keys to read (share_of); k_attend_join brings the parts of a row to the largest reference.
//
// What bounds it, with times on one card (kernel, then join).  4 sequences of 131072 tokens, one query each of 32 heads on 8 kv heads of 128,
// bfloat16: the reads, 2.14 GB in 355 + 5 us, 6.0 TB/s.  32 prefixes of up to 2048 tokens with 8 drafts: 49 + 6 us, 2.2 times the time of its 152 MB; half of it
// is the start (lengths, positions, table, first tile: loads that wait for each other) and the drafts' own keys.  8 prefixes of up to 4096 tokens,
// 8 drafts, 9 queries each: 59 + 10 us for 88 MB and 22 GFLOP; matrix instructions are under way for 17 % of the time, the rest are waits for the
// shared tiles and each other with two waves per SIMD (registers leave no third), and the 48 MB of parts that are written and read.  24 float32 sequences, 5 queries of 14 heads on
// 2 kv heads of 64, window 1000: 20 + 4 us against 2.7 for its bytes: latency of 4 tiles per wave.  One query: 5.9 us, all latency.
#include "specgbv_attend.hpp"

namespace specgbv {
namespace {

// Waves per SIMD, and so workgroups per compute unit, that the registers of a tile, its rows (16 RT) and their sums leave room for.
constexpr int room_for(int DP, int element_bytes, int RT) { return DP == 256 || (element_bytes == 4 && DP == 128 && RT == 2) ? 1 : 2; }

template <typename T, int DP> struct Shape {
    static constexpr bool kBf = sizeof(T) == 2;
    static constexpr int kKeys = kBf ? 32 : 16;              // of a tile
    static constexpr int kRun = kKeys / 4;                   // keys of a lane
    static constexpr int kHalves = kBf ? 2 : 1;
    static constexpr int kPiece = 16 / sizeof(T);            // entries of a 16-byte piece
    static constexpr int kSteps = DP / (4 * kPiece);         // pieces of a key that a lane takes
    static constexpr int kVec = kBf ? (DP >= 128 ? 8 : 4) : 4;   // adjacent entries of a value that a lane takes
    static constexpr int kGroups = DP / (16 * kVec);         // such vectors per key
    static constexpr int kCols = kGroups * kVec;             // result tiles of 16 entries
    static constexpr int waves(int RT) { return room_for(DP, sizeof(T), RT); }
};

// Not 0 where an entry of a 32-bit word is not finite: its exponent's bits, all ones, carry out of it when one is added.
template <typename T> __device__ __forceinline__ uint32_t exponents_full(uint32_t w)
{
    if constexpr (sizeof(T) == 4) return ((w & 0x7FFFFFFFu) + 0x00800000u) & 0x80000000u;
    else return (((w & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u);
}

// One entry's bits against a kind of value that is not finite: 0 not a number, 1 +inf, 2 -inf.
template <typename T> __device__ __forceinline__ bool is_kind(uint32_t e, int kind)
{
    constexpr uint32_t inf = sizeof(T) == 2 ? 0x7F80u : 0x7F800000u, sign = sizeof(T) == 2 ? 0x8000u : 0x80000000u;
    return kind == 0 ? (e & ~sign) > inf : e == (kind == 1 ? inf : (inf | sign));
}

// Asynchronous 16-byte load per lane into LDS bytes [dst + 16 lane, ...), dst the same for the wave; it counts as a vector load.
// (In assembly because the compiler makes every later wait one for all loads once it sees such a load itself.)
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t byte_offset, uint32_t dst)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(byte_offset), "s"(base), "s"(dst) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }

// A barrier that waits for what has been read from LDS, so that it can be written to behind it, but for no load from memory, and that no access
// to memory is moved across.
__device__ __forceinline__ void meet()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <typename T, int DP, int RT, int WK, bool PARTS>
__global__ void __launch_bounds__(kAttendThreads, (Shape<T, DP>::waves(RT))) k_attend(AttendProblem p)
{
    using S = Shape<T, DP>;
    constexpr int kKeys = S::kKeys, kRun = S::kRun, kHalves = S::kHalves, kSteps = S::kSteps, kVec = S::kVec, kGroups = S::kGroups,
                  kCols = S::kCols, kWords = kVec * sizeof(T) / 4;
    // WK = 4: sums to be joined, [4 waves][RT][kGroups][4][kVec / 4][64]; 1: the tiles, [3][keys, values][kKeys][DP]
    constexpr int kPieces = DP / S::kPiece, kHalfTile = kKeys * DP * static_cast<int>(sizeof(T)), kStages = 3;
    constexpr int kFills = kKeys * kPieces / kAttendThreads;  // of a wave, for the keys and again for the values
    __shared__ F4 sh_acc[WK == 4 ? RT * DP * 16 : (WK == 1 ? kStages * 2 * kHalfTile / 16 : 1)];
    __shared__ float sh_m[kWavesPerGroup][RT * 16], sh_l[kWavesPerGroup][RT * 16];
    __shared__ int sh_range[8];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quad = lane >> 4;

    // ---- which rows, which keys.  Row blocks of one item (they read the same keys) are 8 workgroups apart: on one XCD.
    int item, block;
    if constexpr (WK == 0) {                                  // no barrier stands in the way of waves that have nothing to do
        const int at = blockIdx.x * kWavesPerGroup + wave;
        item = p.by_blocks.div(at); block = p.by_blocks.mod(at, item);
        if (item >= p.items) return;
    } else if (p.row_blocks == 1) { item = blockIdx.x; block = 0; }
    else {
        const int set = p.by_blocks.div(blockIdx.x >> 3);
        item = set * 8 + (blockIdx.x & 7); block = p.by_blocks.mod(blockIdx.x >> 3, set);
        if (item >= p.items) return;
    }
    const int rest = p.by_kv_heads.div(item), head0 = p.by_kv_heads.mod(item, rest);
    const int held = static_cast<int>(capacity_of(p.map));
    Share share{rest, 0, 1, rest, 0};
    if (PARTS) {
        share = share_of(p, rest, held, lane);
        if (share.unit < 0) return;                           // (the same for the whole workgroup)
        if (share.part == 0 && head0 == 0 && block == 0 && threadIdx.x == 0) p.places[share.unit] = make_int2(share.at, share.parts);
    }
    const int unit = share.unit, part = share.part;
    const int first = unit * p.drafts;                        // its first sequence
    const int in_draft = p.tokens * p.group, rows = in_draft * p.drafts;
    const int row0 = block * p.block_rows + (WK == 1 ? wave * 16 * RT : 0);
    const int row_end = min(rows, (block + 1) * p.block_rows);

    const int shared = p.shared_len ? max(0, min(p.shared_len[unit], held)) : held;

    // Rows behind the last one take its place (their loads are those of the last row) and are nowhere stored.
    int64_t q_at[RT], out_at[RT];
    int pos[RT], draft[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row0 + r * 16 + col, row_end - 1);
        draft[r] = p.by_in_draft.div(row);
        const int in = p.by_in_draft.mod(row, draft[r]), t = p.by_group.div(in), head = head0 * p.group + p.by_group.mod(in, t), s = first + draft[r];
        pos[r] = p.positions[s * p.positions_stride + t];
        q_at[r] = s * p.q_stride[0] + t * p.q_stride[1] + head * p.q_stride[2];
        if (!PARTS) out_at[r] = s * p.out_stride[0] + t * p.out_stride[1] + head * p.out_stride[2];
    }

    // ---- queries
    U4 qf[RT][kSteps];
    const T *q = static_cast<const T *>(p.q);
    if (p.q_wide) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int e = (4 * i + quad) * S::kPiece;
                qf[r][i] = *reinterpret_cast<const U4 *>(q + q_at[r] + (e < p.head_dim ? e : 0));
            }
    } else {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int e = (4 * i + quad) * S::kPiece;
                const T *src = q + q_at[r] + (e < p.head_dim ? e : 0);
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (S::kBf) w[j] = src[2 * j] | static_cast<uint32_t>(src[2 * j + 1]) << 16;
                    else w[j] = __float_as_uint(src[j]);
                }
                qf[r][i] = U4{w[0], w[1], w[2], w[3]};
            }
    }
    if (p.head_dim != DP) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            if ((4 * i + quad) * S::kPiece >= p.head_dim)
#pragma unroll
                for (int r = 0; r < RT; ++r) qf[r][i] = U4{0, 0, 0, 0};
    }
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

    // ---- the keys: one stretch of the unit's, or each draft's own ones in turn (the waves take the drafts in turn)
    const T *kb = static_cast<const T *>(p.k) + head0 * static_cast<int64_t>(p.k_head_stride);
    const T *vb = static_cast<const T *>(p.v) + head0 * static_cast<int64_t>(p.v_head_stride);
    const int run_k = col >> 2, in_run = col & 3;
    constexpr bool kTurned = S::kBf && WK == 1;               // values come out of LDS turned: entry 16 c + col of the lane's run of keys
    // WK = 1: which bytes of a run this lane brings to LDS, [n]: row (n 64 + lane) / kPieces of the run, piece ^ what spreads the banks
    uint32_t fill_k[WK == 1 ? kFills : 1], fill_v[WK == 1 ? kFills : 1];
    if constexpr (WK == 1) {
#pragma unroll
        for (int n = 0; n < kFills; ++n) {
            const int unit = (wave * kFills + n) * 64 + lane, row = unit / kPieces, slot = unit % kPieces;
            const int of_key = S::kBf ? row >> 3 << 2 | (row & 3) : row;                   // its row in the product
            const int e = (slot ^ (of_key & (kPieces < 16 ? kPieces - 1 : 15))) * S::kPiece, ev = (kTurned ? slot ^ (row & 3) << 1 : slot) * S::kPiece;
            fill_k[n] = static_cast<uint32_t>(row % kRun * p.k_token_stride + (e < p.head_dim ? e : 0)) * static_cast<uint32_t>(sizeof(T));
            fill_v[n] = static_cast<uint32_t>(row % kRun * p.v_token_stride + (ev < p.head_dim ? ev : 0)) * static_cast<uint32_t>(sizeof(T));
        }
    }
    // the drafts' own keys, behind the shared ones: the unit's parts take the drafts in turn, and so do their waves where they share the rows
    const int last_row = min((block + 1) * p.block_rows, rows) - 1;
    const int own_from = WK == 4 ? 4 * part : p.by_in_draft.div(block * p.block_rows) + part;
    const int own_to = !PARTS || !p.shared_len ? 0 : (WK == 4 ? p.drafts : p.by_in_draft.div(last_row) + 1);    // (drafts with rows in this workgroup)
    const int own_step = WK == 4 ? 4 * share.parts : share.parts;
    bool any = own_from < own_to;                             // something may have been summed
    bool vast = false;                                        // a row of this wave has a reference beyond 2^20 (its neighbours' products are then rounded by themselves too)
#pragma unroll 1
    for (int seg = -1; seg < own_to; seg = seg < 0 ? own_from + (WK == 4 ? wave : 0) : seg + own_step) {
    const bool own = seg >= 0;                                // -1: what the unit's sequences share
    const int step = WK == 4 && !own ? 4 * kKeys : kKeys;
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
    const bool active = lo_all < hi_all;                      // this wave has rows that see something
    if (WK == 1) {
        __syncthreads();                                      // (and nobody reads the tiles of what was before any longer)
        if (lane == 0) { sh_range[wave] = lo_all; sh_range[4 + wave] = hi_all; }
        __syncthreads();
        lo_all = __builtin_amdgcn_readfirstlane(min(min(sh_range[0], sh_range[1]), min(sh_range[2], sh_range[3])));
        hi_all = __builtin_amdgcn_readfirstlane(max(max(sh_range[4], sh_range[5]), max(sh_range[6], sh_range[7])));
    }
    int start = lo_all >= hi_all ? 0 : lo_all / kKeys * kKeys, end = lo_all >= hi_all ? 0 : hi_all;
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
    int tile = start + (WK == 4 && !own ? wave * kKeys : 0);

    // The places of a tile's four runs of keys: page_size is a multiple of a run, and so is where a tile starts.  Runs behind the last key
    // take the last one's place, so that nothing is read outside pages that hold keys; their scores are masked.  All of it is the same for
    // the whole wave and goes through scalar loads, which do not queue behind the keys and values on their way.
    struct Pages { int page[4]; };
    const ConstTable row_table = reinterpret_cast<ConstTable>(reinterpret_cast<uintptr_t>(p.map.table + sequence * p.map.table_stride));
    auto run_key = [&](int t, int r) { return min(t + r * kRun, (end - 1) / kRun * kRun); };
    auto pages_of = [&](int t) {                              // as they stand in the table: nothing waits for them here
        Pages at;
#pragma unroll
        for (int r = 0; r < 4; ++r) at.page[r] = row_table[p.map.page.div(run_key(t, r))];
        return at;
    };
    auto run_of = [&](const Pages &at, int t, int run) {
        int page[4], slot[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int key = run_key(t, r);
            page[r] = static_cast<uint32_t>(at.page[r]) < static_cast<uint32_t>(p.map.pages) ? at.page[r] : -1;
            slot[r] = p.map.page.mod(key, p.map.page.div(key));
        }
        const bool odd = run & 1, upper = run & 2;
        const int p0 = odd ? page[1] : page[0], p1 = odd ? page[3] : page[2];
        const int s0 = odd ? slot[1] : slot[0], s1 = odd ? slot[3] : slot[2];
        return Place{upper ? p1 : p0, upper ? s1 : s0};
    };
    U4 kf[kHalves][kSteps];
    uint32_t vf[kRun][kGroups][kWords];
    // (`there` false: the loads go to one line and nobody uses them.  They are issued all the same, or the waits for what was loaded
    // before them would have to allow for their absence and wait for everything.)
    auto load_keys = [&](Place at, bool there) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            const int64_t off = max(at.page, 0) * static_cast<int64_t>(p.k_page_stride) + (at.slot + 4 * h + in_run) * static_cast<int64_t>(p.k_token_stride);
            const T *src = kb + (there ? off : 0);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int e = (4 * i + quad) * S::kPiece;
                kf[h][i] = *reinterpret_cast<const U4 *>(src + (e < p.head_dim ? e : 0));
            }
        }
    };
    auto load_values = [&](Place at, bool there) {
        const int64_t off = max(at.page, 0) * static_cast<int64_t>(p.v_page_stride) + at.slot * static_cast<int64_t>(p.v_token_stride);
        const T *src = vb + (there ? off : 0);
        const int64_t next_key = there ? p.v_token_stride : 0;
#pragma unroll
        for (int k = 0; k < kRun; ++k)
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int e = (g * 16 + col) * kVec;
                struct alignas(4 * kWords) Words { uint32_t w[kWords]; };
                const Words v = *reinterpret_cast<const Words *>(src + k * next_key + (e < p.head_dim ? e : 0));
#pragma unroll
                for (int w = 0; w < kWords; ++w) vf[k][g][w] = v.w[w];
            }
    };

    // the tile at t into stage `to` of LDS: a run of keys by each wave, so that what differs between the lanes stays the same for all tiles
    auto fill = [&](int table_page, int t, int to) {
        const int key = run_key(t, wave);
        const int64_t page = static_cast<uint32_t>(table_page) < static_cast<uint32_t>(p.map.pages) ? table_page : 0;
        const int64_t slot = p.map.page.mod(key, p.map.page.div(key));
        const T *keys = kb + page * p.k_page_stride + slot * p.k_token_stride, *values = vb + page * p.v_page_stride + slot * p.v_token_stride;
        const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(sh_acc)) + to * 2 * kHalfTile + wave * kFills * 1024;
#pragma unroll
        for (int n = 0; n < kFills; ++n) {
            load_to_lds(keys, fill_k[n], base + n * 1024);
            load_to_lds(values, fill_v[n], base + kHalfTile + n * 1024);
        }
    };
    auto own_page = [&](int t) { return row_table[p.map.page.div(run_key(t, wave))]; };
    auto read_keys = [&](int from) {
        const char *base = reinterpret_cast<const char *>(sh_acc) + from * 2 * kHalfTile;
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int slot = (4 * i + quad) ^ (col & (kPieces < 16 ? kPieces - 1 : 15));
                kf[h][i] = *reinterpret_cast<const U4 *>(base + ((run_k * kRun + 4 * h + in_run) * kPieces + slot) * 16);
            }
    };
    U4 va[kTurned ? kCols : 1];                               // kTurned: eight keys' entries 16 c + col
    auto read_values = [&](int from) {
        const char *base = reinterpret_cast<const char *>(sh_acc) + from * 2 * kHalfTile + kHalfTile;
        if constexpr (kTurned) {
            // 16 lanes read 4 keys of 16 entries, four entries each, and get one entry of the 4 keys each
            typedef short S4 __attribute__((ext_vector_type(4)));
            typedef S4 __attribute__((address_space(3))) *Turn;
            const int spread = col >> 2;
            const char *mine = base + (quad * kRun + spread) * DP * 2 + (col & 3) * 8;
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const char *at = mine + ((c & 3) ^ spread) * 32 + (c & ~3) * 32;
                const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Turn)(uint32_t)(uintptr_t)at);
                const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Turn)(uint32_t)(uintptr_t)(at + 4 * DP * 2));
                __builtin_memcpy(&va[c].x, &lo, 8);
                __builtin_memcpy(&va[c].z, &hi, 8);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kRun; ++k)
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    struct alignas(4 * kWords) Words { uint32_t w[kWords]; };
                    const Words v = *reinterpret_cast<const Words *>(base + ((quad * kRun + k) * DP + (g * 16 + col) * kVec) * static_cast<int>(sizeof(T)));
#pragma unroll
                    for (int w = 0; w < kWords; ++w) vf[k][g][w] = v.w[w];
                }
        }
    };
    // bfloat16: one entry of the lane's eight keys, the left operand of the second product
    auto entry_of = [&](int c) {
        if constexpr (kTurned) return va[c];
        else {
            const int g = c / kVec, j = c % kVec;
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = __builtin_amdgcn_perm(vf[2 * k + 1][g][j / 2], vf[2 * k][g][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
            return U4{w[0], w[1], w[2], w[3]};
        }
    };
    auto without_odd = [](uint32_t x) {                       // entries that are not finite made 0
        if (S::kBf) {
            if ((x & 0x7F80u) == 0x7F80u) x &= 0xFFFF0000u;
            if ((x & 0x7F800000u) == 0x7F800000u) x &= 0x0000FFFFu;
            return x;
        }
        return (x & 0x7F800000u) == 0x7F800000u ? 0u : x;
    };

    Pages next{};
    Place here_v{-1, 0};
    int stage = 0;                                            // of the tile at hand
    int next_page = 0;                                        // WK = 1: of this wave's run two tiles on
    bool bad_pages = false;                                   // WK = 1: some page between start and end is not there
    if (tile < end) {
        if constexpr (WK != 1) {
            const Pages at = pages_of(tile);
            here_v = run_of(at, tile, quad);
            load_keys(run_of(at, tile, run_k), true);
            load_values(here_v, true);
            next = pages_of(tile + step);                     // (behind the end: the last run's page)
        } else {
            const int first_page = own_page(tile), second = own_page(tile + step);
            next_page = own_page(tile + 2 * step);
            uint32_t bad = 0;                                 // (in front of the fills, which a wait for these loads would wait for too)
            for (int n = p.map.page.div(start) + lane, last = p.map.page.div(end - 1); n <= last; n += 64)
                bad |= static_cast<uint32_t>(p.map.table[sequence * p.map.table_stride + n]) < static_cast<uint32_t>(p.map.pages) ? 0u : 1u;
            bad_pages = __any(bad != 0);
            fill(first_page, tile, 0);
            if (tile + step < end) fill(second, tile + step, 1);
        }
    }
    bool odd = false;                                         // a value that is not finite was cleared
    for (; tile < end; tile += step) {
        const bool more = tile + step < end;
        const int here = stage;
        bool lost_here = false;                               // WK = 1: the lane's run has no page
        if constexpr (WK == 1) {
            if (more) wait_for_loads<2 * kFills>();           // this tile is there, the next one may be on its way
            else wait_for_loads<0>();
            meet();                                           // for all waves, and nobody reads the tile before it any longer
            stage = stage == kStages - 1 ? 0 : stage + 1;
            if (tile + 2 * step < end) {
                fill(next_page, tile + 2 * step, stage == kStages - 1 ? 0 : stage + 1);
                next_page = own_page(tile + 3 * step);
            }
            if (!active) continue;                            // uniform
            read_keys(here);
            if (bad_pages) lost_here = run_of(pages_of(tile), tile, quad).page < 0;
        }
        // scores: keys x rows
        F4 s[RT][kHalves];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < kHalves; ++h) s[r][h] = F4{0, 0, 0, 0};
        if (p.head_dim != DP) {
            int mine = quad;
            asm volatile("" : "+v"(mine));                    // (the comparisons stay here: kept over the loop they cost scalar registers)
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                if ((4 * i + mine) * S::kPiece >= p.head_dim)
#pragma unroll
                    for (int h = 0; h < kHalves; ++h) kf[h][i] = U4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    if constexpr (S::kBf)
                        s[r][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, kf[h][i]), __builtin_bit_cast(B8, qf[r][i]), s[r][h], 0, 0, 0);
                    else {
                        const F4 a = __builtin_bit_cast(F4, kf[h][i]), b = __builtin_bit_cast(F4, qf[r][i]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[r][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], s[r][h], 0, 0, 0);
                    }
                }
        const Place cur_v = here_v;
        if constexpr (WK != 1) {
            __builtin_amdgcn_sched_barrier(0);
            load_keys(run_of(next, tile + step, run_k), more);
            here_v = run_of(next, tile + step, quad);
            next = pages_of(tile + 2 * step);
            __builtin_amdgcn_sched_barrier(0);
        } else read_values(here);

        // weights
        const bool lost = WK != 1 ? cur_v.page < 0 : lost_here;
        const bool partial = tile < lo_most || tile + kKeys > hi_least || tile + kKeys > end || (WK != 1 ? __any(lost) : bad_pages);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if (partial) {
                const int base = tile + quad * kRun;
                const int from = max(row_low[r] - base, 0), to = lost ? 0 : min(max(row_high[r] - base, 0), kRun);
#pragma unroll
                for (int k = 0; k < kRun; ++k) s[r][k / 4][k % 4] = k >= from && k < to ? s[r][k / 4][k % 4] : -INFINITY;
            }
            float top = s[r][0][0];
#pragma unroll
            for (int k = 1; k < kRun; ++k) top = fmaxf(top, s[r][k / 4][k % 4]);
            top *= p.c;
            if (__any(top > ref[r] + kRaise)) {
                // (row by row: a reference that one row raises is not the others')
                top = row_largest(top);
                const float now = top > ref[r] + kRaise ? top : ref[r];
                const float f = now == ref[r] ? 1.0f : exp2_of(ref[r] - now);        // (-inf to -inf: nothing summed yet)
                vast = vast || __any(fabsf(now) > 1048576.0f && now != -INFINITY);
                ref[r] = now;
                sum[r] *= f;
#pragma unroll
                for (int c = 0; c < kCols; ++c) acc[r][c] *= f;
            }
            const float m = ref[r] == -INFINITY ? 0.0f : ref[r];
            if (vast) {
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    float x = s[r][k / 4][k % 4] * p.c;
                    asm volatile("" : "+v"(x));                // (rounded by itself)
                    s[r][k / 4][k % 4] = exp2_of(x - m);
                }
            } else {
#pragma unroll
                for (int k = 0; k < kRun; ++k) s[r][k / 4][k % 4] = exp2_of(fmaf(s[r][k / 4][k % 4], p.c, -m));
            }
#pragma unroll
            for (int k = 0; k < kRun; ++k) sum[r] += s[r][k / 4][k % 4];
        }

        // values that some rows do not see: a weight of 0 does not take out what is not finite.  In such tiles keys that no row sees are
        // cleared, and so is what is not finite; it is put back behind the loop, for the rows that see it.
        if (partial) {
            const int base = tile + quad * kRun;
            uint32_t bad = 0, keep[kRun];
#pragma unroll
            for (int k = 0; k < kRun; ++k) keep[k] = lost | (base + k < lo_all) | (base + k >= hi_all) ? 0u : 0xFFFFFFFFu;
            auto clean = [&](uint32_t &w, uint32_t mask) { w &= mask; bad |= exponents_full<T>(w); };
            if constexpr (kTurned) {
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    clean(va[c].x, (keep[0] & 0xFFFFu) | (keep[1] & 0xFFFF0000u));
                    clean(va[c].y, (keep[2] & 0xFFFFu) | (keep[3] & 0xFFFF0000u));
                    clean(va[c].z, (keep[4 % kRun] & 0xFFFFu) | (keep[5 % kRun] & 0xFFFF0000u));
                    clean(va[c].w, (keep[6 % kRun] & 0xFFFFu) | (keep[7 % kRun] & 0xFFFF0000u));
                }
            } else {
#pragma unroll
                for (int k = 0; k < kRun; ++k)
#pragma unroll
                    for (int g = 0; g < kGroups; ++g)
#pragma unroll
                        for (int w = 0; w < kWords; ++w) clean(vf[k][g][w], keep[k]);
            }
            if (__any(bad != 0)) {
                odd = true;
                if constexpr (kTurned) {
#pragma unroll
                    for (int c = 0; c < kCols; ++c) va[c] = U4{without_odd(va[c].x), without_odd(va[c].y), without_odd(va[c].z), without_odd(va[c].w)};
                } else {
#pragma unroll
                    for (int k = 0; k < kRun; ++k)
#pragma unroll
                        for (int g = 0; g < kGroups; ++g)
#pragma unroll
                            for (int w = 0; w < kWords; ++w) vf[k][g][w] = without_odd(vf[k][g][w]);
                }
            }
        }

        // sums of values: entries x rows.  bfloat16 values meet weights rounded to bfloat16, the one pair the matrix instructions take (a product in float32
        // has an eighth of their rate): results are off by 0.0018 to 0.0024 of themselves against 64 bits where their own rounding makes 0.0017 (root mean
        // square, 40 to 16384 keys).  The sum of weights has them unrounded; the rounded ones there change this in the third digit only.
        if constexpr (S::kBf) {
            B8 w[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int k = 0; k < kRun; ++k) w[r][k] = static_cast<__bf16>(s[r][k / 4][k % 4]);
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const U4 a = entry_of(c);
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a), w[r], acc[r][c], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int k = 0; k < kRun; ++k)
                        acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[k][c / kVec][c % kVec]), s[r][0][k], acc[r][c], 0, 0, 0);
        }
        if constexpr (WK != 1) load_values(here_v, more);
    }
    // ---- what was not finite in tiles that not all rows see whole: products of marks alone say which rows see such an entry
    if (odd) {
#pragma unroll 1
        for (int again = start + (WK == 4 && !own ? wave * kKeys : 0); again < end; again += step) {
            const Place at = run_of(pages_of(again), again, quad);
            if (again >= lo_most && again + kKeys <= hi_least && again + kKeys <= end && !(WK != 1 ? __any(at.page < 0) : bad_pages)) continue;
            const int base = again + quad * kRun;
            uint32_t seen[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int from = max(row_low[r] - base, 0), to = at.page < 0 ? 0 : min(max(row_high[r] - base, 0), kRun);
                seen[r] = from < to ? ((1u << to) - 1) & ~((1u << from) - 1) : 0u;
            }
            const T *src = vb + max(at.page, 0) * static_cast<int64_t>(p.v_page_stride) + at.slot * static_cast<int64_t>(p.v_token_stride);
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int d = kTurned ? 16 * c + col : (c / kVec * 16 + col) * kVec + c % kVec;
                uint32_t e[kRun];
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    const T x = src[k * static_cast<int64_t>(p.v_token_stride) + (d < p.head_dim ? d : 0)];
                    if constexpr (S::kBf) e[k] = x;
                    else e[k] = __float_as_uint(x);
                }
#pragma unroll 1
                for (int kind = 0; kind < 3; ++kind) {
                    const float what = kind == 0 ? NAN : (kind == 1 ? INFINITY : -INFINITY);
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        F4 n{0, 0, 0, 0};
                        if constexpr (S::kBf) {
                            B8 a, b;
#pragma unroll
                            for (int k = 0; k < kRun; ++k) {
                                a[k] = static_cast<__bf16>(is_kind<T>(e[k], kind) ? 1.0f : 0.0f);
                                b[k] = static_cast<__bf16>(seen[r] >> k & 1 ? 1.0f : 0.0f);
                            }
                            n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, n, 0, 0, 0);
                        } else {
#pragma unroll
                            for (int k = 0; k < kRun; ++k)
                                n = __builtin_amdgcn_mfma_f32_16x16x4f32(is_kind<T>(e[k], kind) ? 1.0f : 0.0f, seen[r] >> k & 1 ? 1.0f : 0.0f, n, 0, 0, 0);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (n[i] > 0.0f) acc[r][c][i] += what;
                    }
                }
            }
        }
    }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) sum[r] = row_total(sum[r]);

    // ---- the waves of a workgroup join: each brings its sums to the largest reference, then wave i adds up the entries i of all
    if (WK == 4) {
        if (quad == 0)
#pragma unroll
            for (int r = 0; r < RT; ++r) { sh_m[wave][r * 16 + col] = ref[r]; sh_l[wave][r * 16 + col] = sum[r]; }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float most = -INFINITY, total = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) most = fmaxf(most, sh_m[w][r * 16 + col]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float m = sh_m[w][r * 16 + col];
                total += sh_l[w][r * 16 + col] * (m == most ? 1.0f : exp2_of(m - most));
            }
            const float f = ref[r] == most ? 1.0f : exp2_of(ref[r] - most);
            ref[r] = most; sum[r] = total;
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int n = 0; n < kVec / 4; ++n) {
                        F4 v;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = acc[r][g * kVec + 4 * n + e][i] * f;
                        sh_acc[((((wave * RT + r) * kGroups + g) * 4 + i) * (kVec / 4) + n) * 64 + lane] = v;
                    }
        }
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (row0 + r * 16 + col >= row_end) continue;
        // Partial sums are held in the order in which lanes hold them: in order (kTurned), or vector ((g 4 + i) kVec / 4 + n) 4 + quad of
        // a row are entries (16 g + 4 quad + i) kVec + 4 n + 0..3.  Where nothing was summed they are not written: the sum of weights says so.
        const float inv = sum[r] != 0.0f ? 1.0f / sum[r] : 0.0f;
        const int64_t at = PARTS ? (static_cast<int64_t>(share.at + part) * p.kv_heads + head0) * rows + row0 + r * 16 + col : 0;
        if (PARTS && (WK != 4 || wave == 0) && quad == 0) p.ml[at] = make_float2(ref[r], sum[r]);
        if (PARTS && !any) continue;
        if constexpr (kTurned) {                              // result c of a lane is entries 16 c + 4 quad + 0..3
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int d = 16 * c + 4 * quad;
                if (PARTS) reinterpret_cast<F4 *>(p.acc + at * DP)[d / 4] = acc[r][c];
                else if (d < p.head_dim) store_entries(static_cast<T *>(p.out) + out_at[r] + d, acc[r][c], pos[r] < 0 ? 0.0f : inv, p.out_wide);
            }
            continue;
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (WK == 4 && i != wave) continue;
                const int d = (16 * g + 4 * quad + i) * kVec;
#pragma unroll
                for (int n = 0; n < kVec / 4; ++n) {
                    F4 v{0, 0, 0, 0};
                    if (WK == 4) {
#pragma unroll
                        for (int w = 0; w < 4; ++w) v += sh_acc[((((w * RT + r) * kGroups + g) * 4 + i) * (kVec / 4) + n) * 64 + lane];
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = acc[r][g * kVec + 4 * n + e][i];
                    }
                    if (PARTS) reinterpret_cast<F4 *>(p.acc + at * DP)[((g * 4 + i) * (kVec / 4) + n) * 4 + quad] = v;
                    else if (d + 4 * n < p.head_dim)
                        store_entries(static_cast<T *>(p.out) + out_at[r] + d + 4 * n, v, pos[r] < 0 ? 0.0f : inv, p.out_wide);
                }
            }
    }
}

template <typename T, int DP, int RT, int WK, bool PARTS>
hipError_t launch_one(AttendProblem p, hipStream_t stream)
{
    p.items = p.all_parts * p.kv_heads;
    p.by_blocks = Divider::of(p.row_blocks);
    const int64_t grid = WK == 0 ? (static_cast<int64_t>(p.items) * p.row_blocks + kWavesPerGroup - 1) / kWavesPerGroup : p.row_blocks == 1 ? p.items : static_cast<int64_t>((p.items + 7) / 8 * 8) * p.row_blocks;
    if (grid >= kLaunchGroups) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_attend<T, DP, RT, WK, PARTS>), dim3(static_cast<unsigned>(grid)), dim3(kAttendThreads), 0, stream, p);
    return hipGetLastError();
}

template <typename T, int DP, bool PARTS>
hipError_t launch_rows(const AttendProblem &p, hipStream_t stream)
{
    const int rows = p.tokens * p.group * p.drafts;
    constexpr int RT = DP < 256 ? 2 : 1;
    if constexpr (!PARTS)
        if (p.lone) return rows <= 16 ? launch_one<T, DP, 1, 0, false>(p, stream) : launch_one<T, DP, RT, 0, false>(p, stream);
    if (rows <= 16) return launch_one<T, DP, 1, 4, PARTS>(p, stream);
    return p.few ? launch_one<T, DP, RT, 4, PARTS>(p, stream) : launch_one<T, DP, RT, 1, PARTS>(p, stream);
}

template <typename T, int DP>
hipError_t launch_typed(AttendProblem p, hipStream_t stream)
{
    p.in_order = Shape<T, DP>::kBf && !p.few;
    if (p.all_parts == p.units && !p.ml) return launch_rows<T, DP, false>(p, stream);
    if (join_grid<DP>(p) >= kLaunchGroups) return hipErrorInvalidConfiguration;
    const hipError_t e = launch_rows<T, DP, true>(p, stream);
    return e != hipSuccess ? e : launch_join<T, DP, Shape<T, DP>::kVec>(p, stream);
}

template <typename T>
hipError_t launch_dim(const AttendProblem &p, hipStream_t stream)
{
    if (p.head_dim <= 64) return launch_typed<T, 64>(p, stream);
    if (p.head_dim <= 128) return launch_typed<T, 128>(p, stream);
    return launch_typed<T, 256>(p, stream);
}

}  // namespace

static AttendPlan plan_for(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                           int64_t longest)
{
    AttendPlan a{};
    a.drafts = drafts; a.shared = shared;
    const int dp = head_dim <= 64 ? 64 : (head_dim <= 128 ? 128 : 256);
    const int rows = tokens * (heads / kv_heads) * drafts, tall = dp < 256 ? 32 : 16;
    // rows of a workgroup: a wave's, which all four share, or four waves' own ones, spread evenly over the workgroups
    // Up to here the waves of a workgroup share its rows and take the keys in turn; beyond they share the keys.  Sharing the rows keeps the keys out of
    // LDS and needs no barrier, but each 32 rows load them again, and drafts' own keys meet all rows of a workgroup.  Shared rows / shared keys, us, bfloat16,
    // 2 kv heads of 128: 16 sequences of up to 2048 tokens 24 / 29 at 144 rows, 27 / 40 at 256, 54 / 43 at 544; heads of 256: 42 / 38 at 72 rows, 57 / 47 at 144;
    // prefixes of 8 drafts (8 kv heads) 46 / 52 at 96 rows, 92 / 74 at 288; of 4 drafts 61 / 52 at 144; float32, 8 sequences of up to 4096, 35 / 43 at 144, 139 / 86 at 544.
    const int few_rows = dp == 256 ? 64 : (shared ? 128 : 256);
    a.few = rows <= few_rows;
    if (a.few) a.block_rows = rows <= 16 ? 16 : tall;
    else {
        const int blocks = (rows + 4 * tall - 1) / (4 * tall), waves = (rows + tall - 1) / tall;
        a.block_rows = (waves + blocks - 1) / blocks * tall;
    }
    a.row_blocks = (rows + a.block_rows - 1) / a.block_rows;
    a.units = sequences / drafts;
    a.all_parts = a.units;
    if (window > 0) longest = longest < static_cast<int64_t>(window) + tokens ? longest : static_cast<int64_t>(window) + tokens;
    const int64_t base = static_cast<int64_t>(a.units) * kv_heads * a.row_blocks;
    // Keys of a part at least.  One sequence of 1000 tokens, 8 heads on 2 kv heads, 128 / 256 / 512, us: 10.4 / 11.1 / 13.3 with one query; two of 20000
    // 18.5 / 18.4 / 16.2.  With 36 rows more queries a kv head, 64 / 128 / 256: 12.9 / 14.6 / 18.4, and 20.7 / 19.5 / 21.2 for four of 4096.
    const int least = a.few ? 256 : 128;
    // Workgroups on the card at once.  One / two a compute unit, us: 8 prefixes of 8 drafts with 9 tokens each, 8 kv heads of 128, bfloat16 (room for two)
    // 126 / 69; 16 sequences of up to 2048 tokens, 5 queries each of 16 heads on 4 kv heads of 256 (room for one) 33 / 40, and 33 / 43 in float32 of 128.
    const int64_t slots = static_cast<int64_t>(compute_units()) * room_for(dp, element_bytes, a.block_rows == 16 || dp == 256 ? 1 : 2);
    int64_t chunks = slots / (base < 1 ? 1 : base);
    const int64_t most = (longest + least - 1) / least;
    if (chunks > most) chunks = most;
    if (chunks > kMaxParts) chunks = kMaxParts;
    if (chunks < 1) chunks = 1;
    if (chunks == 1 && !shared) {                              // one pass, nothing to join
        // Few tiles, and more workgroups than the card holds at once: each wave by itself, which saves turns and the join in LDS.  Workgroups / waves, us, one
        // query of 32 heads on 8 kv heads of 128, bfloat16: 256 sequences of up to 40 tokens 18.4 / 13.3, 100 22.3 / 18.0, 200 33.5 / 32.8; 8 sequences (64
        // workgroups) 5.8 / 6.8, 6.1 / 8.7, 7.0 / 12.0.  With many registers a wave, which leave few waves to cover a workgroup's end, up to longer: 9 queries each
        // of 64 sequences 25 / 18 at 40, 36 / 29 at 440, 41 / 38 at 640, in float32 93 / 83 and 108 / 113; one query at heads of 256, 256 sequences 56 / 27, 125 / 120, 156 / 159.
        a.lone = a.few && longest <= (dp == 256 || (dp == 128 && a.block_rows > 16) ? 448 : 208) && base > slots;
        return a;
    }
    a.own_keys = shared ? drafts * 32 : 0;
    a.chunk_keys = least;
    a.grain = !a.few ? 32 : (element_bytes == 2 ? 128 : 64);   // a tile for each wave that takes keys
    a.balanced = a.units <= 64 && (shared || tokens <= 64);
    if (a.balanced) {
        a.most_parts = static_cast<int>(slots / (static_cast<int64_t>(kv_heads) * a.row_blocks));
        if (a.most_parts < a.units) a.most_parts = a.units;
        if (a.most_parts > kMaxParts) a.most_parts = kMaxParts;
        a.all_parts = a.most_parts + a.units;
    } else {
        a.chunks = static_cast<int>(chunks);
        a.all_parts = a.units * a.chunks;
        a.chunk_keys = static_cast<int>(((longest + chunks - 1) / chunks + 127) / 128 * 128);
    }
    const size_t parts = static_cast<size_t>(a.all_parts) * kv_heads * rows;
    a.places_bytes = (static_cast<size_t>(a.units) * sizeof(int2) + 255) / 256 * 256;
    a.ml_bytes = (parts * sizeof(float2) + 255) / 256 * 256;
    a.bytes = a.places_bytes + a.ml_bytes + (parts * dp * sizeof(float) + 255) / 256 * 256;
    return a;
}

// Drafts that share short prefixes are sequences like others: what they have of their own would be most of the work, in units with rows
// of many drafts, and a read once more comes from the L2 caches.  Shared / alone, us: 32 prefixes of 8 drafts, a token each (32 heads, 8 kv heads
// of 128, bfloat16) 24 / 12 at 40 tokens, 24 / 21 at 160, 29 / 29 at 320, 27 / 44 at 640; 8 of 8, 9 tokens each, 31 / 17 at 40, 40 / 34 at 640,
// 46 / 53 at 1280; one of 8, a token each (21 heads, 3 kv heads of 128, float32) 18 / 7 at 40, 26 / 16 at 1280, 26 / 25 at 2560.
// Up to which length they are taken by themselves:
static int64_t alone_up_to(int sequences, int kv_heads, int head_dim, int element_bytes)
{
    const int64_t reads = (int64_t{128} << 20) / (2 * static_cast<int64_t>(sequences) * kv_heads * head_dim * element_bytes);
    return reads < 1024 ? reads : 1024;
}

// (a call asks for the workspace of either way)
AttendPlan plan_attend(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                       int64_t longest)
{
    const AttendPlan plan = plan_for(sequences, drafts, shared, tokens, heads, kv_heads, head_dim, element_bytes, window, longest);
    if (!shared || longest > alone_up_to(sequences, kv_heads, head_dim, element_bytes)) return plan;
    AttendPlan alone = plan_for(sequences, 1, false, tokens, heads, kv_heads, head_dim, element_bytes, window, longest);
    if (alone.bytes < plan.bytes) alone.bytes = plan.bytes;
    return alone;
}

// The parts of a plan, and so its bytes, do not get fewer with the length: the longest one of each way asks for most.
size_t attend_bytes(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                    int64_t held)
{
    const size_t whole = plan_for(sequences, drafts, shared, tokens, heads, kv_heads, head_dim, element_bytes, window, held).bytes;
    const int64_t near = shared ? alone_up_to(sequences, kv_heads, head_dim, element_bytes) : 0;
    if (near < 1) return whole;
    const size_t alone = plan_for(sequences, 1, false, tokens, heads, kv_heads, head_dim, element_bytes, window, near < held ? near : held).bytes;
    return alone > whole ? alone : whole;
}

hipError_t launch_attend(const AttendProblem &p, int dtype, hipStream_t stream)
{
    return dtype == 1 ? launch_dim<uint16_t>(p, stream) : launch_dim<float>(p, stream);
}

}  // namespace specgbv
