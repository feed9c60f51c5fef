// Attention over a cache held in 4 bits: which rows, waves and parts a call is cut into.
#include "specgbv_packed_attend.hpp"

namespace specgbv {

struct AttendShape { int sequences, drafts; bool shared; int tokens, heads, kv_heads, head_dim, element_bytes, window; };
static int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : (head_dim <= 128 ? 128 : 256); }
static int64_t seen_of(const AttendShape &c, int64_t longest)
{
    const int64_t most = static_cast<int64_t>(c.window) + c.tokens;
    return c.window > 0 && longest > most ? most : longest;
}

// Tiles of 16 rows that a wave takes, where there is a choice.  More rows decode and read a tile's keys for more products, but fill fewer workgroups, leave fewer waves a SIMD and more rows empty.
// A workgroup's time is taken as that of so many tokens at the start and a factor on the tokens, the card's as the mean of the workgroups' turns, rounded up and not.  1 / 2 / 4 tiles, us,
// heads of 128 (8 kv heads but where said): 16 sequences of 36 rows 9.9 / 10.5 / 14.4 at 256 tokens, 27.7 / 23.5 / 31.1 at 2048; 64 of them 24.5 / 24.0 / 24.3, 62 / 66 / 59 and at 4096 118 / 123 / 101; 54
// of 72 on 3 kv heads 15.3 / 15.6 / 21.0, 42.5 / 37.1 / 54.2; one of 4000 27.5 / 29.2 / 34.8, 71 / 65 / 76 and at 4096 121 / 118 / 131; 8 prefixes with 288 rows 58.0 / 58.7 / 62.1 at 2048, 92 / 90 / 96 at 4096; 32 of
// them 115 / 110 / 104 at 1024, 284 / 254 / 231 at 4096; heads of 64, 64 sequences of 68 rows 8.6 / 9.1 / 11.0 and 25.3 / 25.0 / 28.8.
static int tiles_of(const AttendShape &c, int64_t longest)
{
    const int rows = c.tokens * (c.heads / c.kv_heads) * c.drafts, tall = rows_tall(c.element_bytes, padded_dim(c.head_dim));
    const int64_t seen = seen_of(c, longest), own = c.shared ? 600 : 0, units = compute_units();
    int best = 1;
    double least = INFINITY;
    for (int tiles = 1; tiles <= tall; tiles *= 2) {
        const int64_t blocks = (rows + 16 * tiles - 1) / (16 * tiles), groups = c.sequences / c.drafts * static_cast<int64_t>(c.kv_heads) * blocks;
        const int64_t start = tiles == 1 ? 450 : (tiles == 2 ? 900 : 1900), tenths = tiles == 1 ? 10 : (tiles == 2 ? 16 : (c.shared || blocks <= 2 ? 28 : 33));
        const double cost = static_cast<double>((groups + units - 1) / units * units + groups) * static_cast<double>(10 * (start + own) + tenths * seen);
        if (cost < least) { least = cost; best = tiles; }
        if (blocks == 1) break;                                // (more would be empty)
    }
    return best;
}

// in_parts: the plan that needs most workspace.
static AttendPlan plan_for(const AttendShape &c, int64_t longest, int RT, bool in_parts = false)
{
    const int drafts = c.drafts, tokens = c.tokens, kv_heads = c.kv_heads, element_bytes = c.element_bytes;
    const bool shared = c.shared;
    AttendPlan a{};
    a.drafts = drafts; a.shared = shared;
    const int dp = padded_dim(c.head_dim);
    const int rows = tokens * (c.heads / kv_heads) * drafts;
    a.block_rows = 16 * RT;
    a.row_blocks = (rows + a.block_rows - 1) / a.block_rows;
    a.units = c.sequences / drafts;
    a.all_parts = a.units;
    longest = seen_of(c, longest);
    const int64_t base = static_cast<int64_t>(a.units) * kv_heads * a.row_blocks;             // stretches of rows with keys of their own
    a.few = kWavesPerGroup;                                    // (that share a workgroup's rows; 0: none do)
    const int64_t slots = static_cast<int64_t>(compute_units()) * packed_waves(element_bytes, dp, RT);      // workgroups on the card at once
    // Keys of a part at least.  128 / 256 / 512, us: one query of 32 heads on 8 kv heads of 128, 10.0 / 10.7 / 12.1 at 4000 tokens; 4 sequences, 9 queries (64 rows at once), 22.7 / 20.1 / 21.7 at 2000
    // and 25.4 / 25.5 / 23.1 at 4000; 8 sequences at heads of 256 11.8 / 12.9 / 15.2 at 2000, 14.9 / 13.1 / 15.0 at 4000.
    const int least = RT == 1 && dp <= 128 ? 128 : 256;
    int64_t chunks = slots / (base < 1 ? 1 : base);
    const int64_t most = (longest + least - 1) / least;
    if (chunks > most) chunks = most;
    if (chunks > kMaxParts) chunks = kMaxParts;
    // Parts cost a join, 4 us and more, and pay from a length on that is the greater the fewer there can be.  In one pass / in parts, us: one query of 32 heads 7.1 / 10.0 at 300 tokens,
    // 8.6 / 10.0 at 600, 10.9 / 10.0 at 1000; of 32 sequences 9.2 / 14.0 at 600, 13.7 / 17.4 at 1000, 22.0 / 22.9 at 2000; 4 sequences, 9 queries (64 rows at once), 17.1 / 16.6 at 300, 20.2 / 17.1 at 600;
    // 8 at heads of 256 9.9 / 11.6 at 300, 12.1 / 11.8 at 600; two tiles of rows between these.
    const int64_t one_pass = RT == 4 ? 256 : (RT == 2 || dp == 256 ? 480 : 800);
    if (longest * slots <= one_pass * (slots + 6 * base)) chunks = 1;
    if (chunks < 1) chunks = 1;
    // About a workgroup for each compute unit: one that fills it, and no parts.  Parts / filled, us: 32 sequences, a query of 32 heads on 8 kv heads of 128 (16 waves) 10.8 / 11.6 at 800 tokens,
    // 18.8 / 17.2 at 1600, 29.9 / 25.5 at 3200; 16 of them 17.3 / 14.3 at 1600, 21.7 / 20.6 at 3200; 16 with 20 rows (32 at once, 8 waves) 11.1 / 11.4 at 400, 14.0 / 13.0 at 800, 20.2 / 17.6 at 1600,
    // 25.6 / 26.2 at 3200; 8 float32 sequences, 8 kv heads of 128 (8 waves), 10.4 / 10.3 at 400, 13.2 / 12.1 at 800, 14.9 / 16.6 at 1600.  Drafts that share a prefix: 32 of 8 (a query
    // each, 8 waves) 25.1 / 21.3 at 800, 30.2 / 26.2 at 1600, 39.4 / 36.8 at 3200; 16 of 8 24.4 / 21.9 at 1600, 29.2 / 31.8 at 3200.
    const int wide = packed_wide(element_bytes, dp, RT);
    if (!in_parts && wide > kWavesPerGroup && base <= compute_units() && longest <= 14 * base && longest > (shared ? 0 : (wide == 16 ? 1000 : 600))) {
        a.few = wide;
        return a;
    }
    if (chunks == 1 && !shared) {                              // nothing to join
        // Few tiles, and more workgroups than the card holds at once: each wave by itself, which saves turns and the join in LDS.  Waves / workgroups, us, one query of 256 sequences, 32 heads
        // on 8 kv heads of 128: 10.4 / 14.7 at 40 tokens, 18.6 / 20.8 at 300, 23.7 / 23.5 at 440; at heads of 256 9.2 / 15.6, 21.8 / 23.4, 27.2 / 26.3; of 64 5.7 / 6.7, 8.7 / 8.3 at 200;
        // 36 rows of 256 sequences 52 / 59 at 30, 66 / 72 at 256, 85 / 86 at 512; 32 rows at once, 64 sequences 17.1 / 24.4 at 30, 24.0 / 27.4 at 256, 33.7 / 33.5 at 512, 256 of them 54 / 84, 71 / 100 and 94 / 118.
        // 64 rows at once share them always (64 sequences of 36 rows 25.8 / 24.4 at 40, 51 / 33 at 640).
        const int64_t by_waves = RT == 4 ? 0 : (RT == 2 ? 512 : (dp == 64 ? 128 : 400));
        if (longest <= by_waves && base > slots) a.few = 0;
        return a;
    }
    a.own_keys = shared ? drafts * 32 : 0;
    a.chunk_keys = least;
    a.grain = kWavesPerGroup * kTile;
    a.balanced = a.units <= 64 && (shared || tokens <= 64);
    if (a.balanced) {
        int64_t parts = slots / (static_cast<int64_t>(kv_heads) * a.row_blocks);
        if (parts < a.units) parts = a.units;
        if (parts > kMaxParts) parts = kMaxParts;
        a.most_parts = static_cast<int>(parts);
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

// Drafts that share short prefixes are sequences like others: each reads the prefix again, which in 4 bits is little, and what it has of its own needs no
// turn of its own and nothing is to be joined.  Shared / alone, us: 32 prefixes of 8 drafts, a token each (32 heads, 8 kv heads of 128, bfloat16) 22 / 10 at 40 tokens,
// 23 / 20 at 320, 25 / 24 at 640, 29 / 40 at 1280; 8 of 8, 9 tokens each, 28 / 24 at 40, 45 / 38 at 1280, 55 / 53 at 2560, 69 / 105 at 5120; 16 of 4, 5 tokens each of 10 heads on
// 2 kv heads (float32) 21 / 13 at 40, 35 / 34 at 2560; 4 of 4, 9 tokens each, heads of 256, 18 / 14 at 40, 28 / 26 at 1280, 32 / 36 at 2560; one of 8, a token each, 8 kv heads of 128,
// 14.6 / 14.6 at 2560, 18 / 24 at 10240.  (The shared side has the join of parts in it, also where each prefix is one part, as with 8 of 8 of 9 tokens.)  Up to which length they are taken by themselves:
// Where their prefixes would be taken whole by workgroups that fill a compute unit, up to half of it: 32 of 8 17.9 / 17.9 at 200, 18 / 25 at 400; 16 of 8 15.8 / 14.6 at 400, 16.8 / 21.2 at 800.
static int64_t alone_up_to(int sequences, int kv_heads, int head_dim, bool filled)
{
    const int64_t entries = (head_dim > 128 ? int64_t{1} << 25 : int64_t{1} << 27) / (static_cast<int64_t>(sequences) * kv_heads * head_dim) / (filled ? 2 : 1);
    return entries < 2560 ? entries : 2560;
}

// (a call of drafts asks for the workspace of parts whatever it takes, so that a caller who brings none learns it at any length)
AttendPlan plan_packed_attend(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                              int64_t longest)
{
    AttendShape c{sequences, drafts, shared, tokens, heads, kv_heads, head_dim, element_bytes, window};
    const int tiles = tiles_of(c, longest);
    AttendPlan plan = plan_for(c, longest, tiles);
    if (!shared) return plan;
    const size_t asked = plan_for(c, longest, tiles, true).bytes;
    if (longest <= alone_up_to(sequences, kv_heads, head_dim, plan.few > kWavesPerGroup)) {
        c.drafts = 1; c.shared = false;
        plan = plan_for(c, longest, tiles_of(c, longest));
    }
    if (plan.bytes < asked) plan.bytes = asked;
    return plan;
}

// The parts of a plan in parts, and so its bytes, do not get fewer with the length: the longest one of each way, with each number of rows, asks for most.
size_t packed_attend_bytes(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                           int64_t held)
{
    AttendShape c{sequences, drafts, shared, tokens, heads, kv_heads, head_dim, element_bytes, window};
    const int64_t near = shared ? alone_up_to(sequences, kv_heads, head_dim, false) : 0;
    size_t most = 0;
    for (int way = 0; way < (near < 1 ? 1 : 2); ++way) {
        if (way == 1) { c.drafts = 1; c.shared = false; }
        for (int tiles = 1; tiles <= rows_tall(element_bytes, padded_dim(head_dim)); tiles *= 2) {
            const size_t bytes = plan_for(c, way == 1 && near < held ? near : held, tiles, true).bytes;
            if (bytes > most) most = bytes;
        }
    }
    return most;
}

hipError_t launch_packed_attend(const PackedProblem &p, int dtype, hipStream_t stream)
{
    if (p.a.head_dim <= 64) return launch_packed_attend_64(p, dtype, stream);
    if (p.a.head_dim <= 128) return launch_packed_attend_128(p, dtype, stream);
    return launch_packed_attend_256(p, dtype, stream);
}

}  // namespace specgbv
