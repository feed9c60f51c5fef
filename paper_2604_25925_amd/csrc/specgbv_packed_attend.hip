// Attention over a cache held in 4 bits: which rows, waves and parts a call is cut into.
#include "specgbv_packed_attend.hpp"

namespace specgbv {

// in_parts: the plan that needs most workspace.
static AttendPlan plan_for(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                           int64_t longest, bool in_parts = false)
{
    AttendPlan a{};
    a.drafts = drafts; a.shared = shared;
    const int dp = head_dim <= 64 ? 64 : (head_dim <= 128 ? 128 : 256);
    const int rows = tokens * (heads / kv_heads) * drafts, tall = 16 * rows_tall(element_bytes, dp);
    a.block_rows = rows <= 16 ? 16 : (rows <= 32 && tall > 32 ? 32 : tall);
    a.row_blocks = (rows + a.block_rows - 1) / a.block_rows;
    a.units = sequences / drafts;
    a.all_parts = a.units;
    if (window > 0) longest = longest < static_cast<int64_t>(window) + tokens ? longest : static_cast<int64_t>(window) + tokens;
    const int64_t base = static_cast<int64_t>(a.units) * kv_heads * a.row_blocks;             // stretches of rows with keys of their own
    a.few = kWavesPerGroup;                                    // (that share a workgroup's rows; 0: none do)
    const int RT = a.block_rows / 16;
    const int64_t slots = static_cast<int64_t>(compute_units()) * packed_waves(element_bytes, dp, RT);      // workgroups on the card at once
    // Keys of a part at least.  128 / 256 / 512, us: one query of 32 heads on 8 kv heads of 128, 10.0 / 10.7 / 12.1 at 4000 tokens; 4 sequences, 9 queries, 22.7 / 20.1 / 21.7 at 2000
    // and 25.4 / 25.5 / 23.1 at 4000; 8 sequences at heads of 256 11.8 / 12.9 / 15.2 at 2000, 14.9 / 13.1 / 15.0 at 4000.
    const int least = RT == 1 && dp <= 128 ? 128 : 256;
    int64_t chunks = slots / (base < 1 ? 1 : base);
    const int64_t most = (longest + least - 1) / least;
    if (chunks > most) chunks = most;
    if (chunks > kMaxParts) chunks = kMaxParts;
    // Parts cost a join, 4 us and more, and pay from a length on that is the greater the fewer there can be.  In one pass / in parts, us: one query of 32 heads 7.1 / 10.0 at 300 tokens,
    // 8.6 / 10.0 at 600, 10.9 / 10.0 at 1000; of 32 sequences 9.2 / 14.0 at 600, 13.7 / 17.4 at 1000, 22.0 / 22.9 at 2000; 4 sequences, 9 queries, 17.1 / 16.6 at 300, 20.2 / 17.1 at 600;
    // 24 float32 sequences, 5 queries of 14 heads on 2 kv heads of 64, 10.5 / 13.9 at 300, 16.3 / 16.0 at 1000; 8 at heads of 256 9.9 / 11.6 at 300, 12.1 / 11.8 at 600.
    const int64_t one_pass = RT == 4 ? 256 : (RT == 2 || dp == 256 ? 480 : 800);
    if (longest * slots <= one_pass * (slots + 6 * base)) chunks = 1;
    if (chunks < 1) chunks = 1;
    // About a workgroup for each compute unit: one that fills it, and no parts.  Parts / filled, us: 32 sequences, a query of 32 heads on 8 kv heads of 128 (16 waves) 10.8 / 11.6 at 800 tokens,
    // 18.8 / 17.2 at 1600, 29.9 / 25.5 at 3200; 16 of them 17.3 / 14.3 at 1600, 21.7 / 20.6 at 3200; 16 with 5 queries (8 waves) 11.1 / 11.4 at 400, 14.0 / 13.0 at 800, 20.2 / 17.6 at 1600,
    // 25.6 / 26.2 at 3200; 24 float32 sequences, 5 queries of 14 heads on 2 kv heads of 64, 15.0 / 13.7 at 800, 18.8 / 18.6 at 1600, 22.6 / 28.5 at 3200.  Drafts that share a prefix: 32 of 8 (a query
    // each, 8 waves) 25.1 / 21.3 at 800, 30.2 / 26.2 at 1600, 39.4 / 36.8 at 3200; 16 of 8 24.4 / 21.9 at 1600, 29.2 / 31.8 at 3200.
    const int wide = packed_wide(element_bytes, dp, RT);
    if (!in_parts && wide > kWavesPerGroup && base <= compute_units() && longest <= 14 * base && longest > (shared ? 0 : (wide == 16 ? 1000 : 600))) {
        a.few = wide;
        return a;
    }
    if (chunks == 1 && !shared) {                              // nothing to join
        // Few tiles, and more workgroups than the card holds at once: each wave by itself, which saves turns and the join in LDS.  Waves / workgroups, us, one query of 256 sequences, 32 heads
        // on 8 kv heads of 128: 10.4 / 14.7 at 40 tokens, 18.6 / 20.8 at 300, 23.7 / 23.5 at 440; at heads of 256 9.2 / 15.6, 21.8 / 23.4, 27.2 / 26.3; of 64 5.7 / 6.7, 8.7 / 8.3 at 200;
        // 9 queries of 64 sequences (64 rows a workgroup) 25.8 / 24.4 at 40 and 51 / 33 at 640, in float32 (32 rows) 22 / 49 and 50 / 72.
        const int64_t by_waves = RT == 4 ? 0 : (RT == 2 ? 1024 : (dp == 64 ? 128 : 400));
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
// 14.6 / 14.6 at 2560, 18 / 24 at 10240.  Up to which length they are taken by themselves:
// Where their prefixes would be taken whole by workgroups that fill a compute unit, up to half of it: 32 of 8 17.9 / 17.9 at 200, 18 / 25 at 400; 16 of 8 15.8 / 14.6 at 400, 16.8 / 21.2 at 800.
static int64_t alone_up_to(int sequences, int kv_heads, int head_dim, bool filled)
{
    const int64_t entries = (head_dim > 128 ? int64_t{1} << 25 : int64_t{1} << 27) / (static_cast<int64_t>(sequences) * kv_heads * head_dim) / (filled ? 2 : 1);
    return entries < 2560 ? entries : 2560;
}

// (a call asks for the workspace of either way)
AttendPlan plan_packed_attend(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                              int64_t longest)
{
    const AttendPlan plan = plan_for(sequences, drafts, shared, tokens, heads, kv_heads, head_dim, element_bytes, window, longest);
    if (!shared || longest > alone_up_to(sequences, kv_heads, head_dim, plan.few > kWavesPerGroup)) return plan;
    AttendPlan alone = plan_for(sequences, 1, false, tokens, heads, kv_heads, head_dim, element_bytes, window, longest);
    if (alone.bytes < plan.bytes) alone.bytes = plan.bytes;
    return alone;
}

// The parts of a plan in parts, and so its bytes, do not get fewer with the length: the longest one of each way asks for most.
size_t packed_attend_bytes(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                           int64_t held)
{
    const size_t whole = plan_for(sequences, drafts, shared, tokens, heads, kv_heads, head_dim, element_bytes, window, held, true).bytes;
    const int64_t near = shared ? alone_up_to(sequences, kv_heads, head_dim, false) : 0;
    if (near < 1) return whole;
    const size_t alone = plan_for(sequences, 1, false, tokens, heads, kv_heads, head_dim, element_bytes, window, near < held ? near : held, true).bytes;
    return alone > whole ? alone : whole;
}

hipError_t launch_packed_attend(const PackedProblem &p, int dtype, hipStream_t stream)
{
    if (p.a.head_dim <= 64) return launch_packed_attend_64(p, dtype, stream);
    if (p.a.head_dim <= 128) return launch_packed_attend_128(p, dtype, stream);
    return launch_packed_attend_256(p, dtype, stream);
}

}  // namespace specgbv
