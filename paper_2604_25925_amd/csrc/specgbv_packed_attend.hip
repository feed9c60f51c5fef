// Attention over a cache held in 4 bits: which rows, waves and parts a call is cut into.
#include "specgbv_packed_attend.hpp"

namespace specgbv {

static AttendPlan plan_for(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                           int64_t longest)
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
    a.few = rows <= 1024;
    const int64_t slots = static_cast<int64_t>(compute_units()) * packed_waves(element_bytes, dp, a.block_rows / 16) * (a.few ? 1 : kWavesPerGroup);
    const int least = a.few ? 256 : 128;
    int64_t chunks = slots / (base < 1 ? 1 : base);
    const int64_t most = (longest + least - 1) / least;
    if (chunks > most) chunks = most;
    if (chunks > kMaxParts) chunks = kMaxParts;
    if (chunks < 1) chunks = 1;
    if (chunks == 1 && !shared) {                              // one pass, nothing to join
        if (a.few && longest <= 208 && base > slots) a.few = 0;        // few tiles, and more workgroups than the card holds at once: each wave by itself
        return a;
    }
    a.own_keys = shared ? drafts * 32 : 0;
    a.chunk_keys = least;
    a.grain = a.few ? kWavesPerGroup * kTile : kTile;
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

AttendPlan plan_packed_attend(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                              int64_t longest)
{
    return plan_for(sequences, drafts, shared, tokens, heads, kv_heads, head_dim, element_bytes, window, longest);
}

// The parts of a plan, and so its bytes, do not get fewer with the length: the longest one of each way asks for most.
size_t packed_attend_bytes(int sequences, int drafts, bool shared, int tokens, int heads, int kv_heads, int head_dim, int element_bytes, int window,
                           int64_t held)
{
    return plan_for(sequences, drafts, shared, tokens, heads, kv_heads, head_dim, element_bytes, window, held).bytes;
}

hipError_t launch_packed_attend(const PackedProblem &p, int dtype, hipStream_t stream)
{
    if (p.a.head_dim <= 64) return launch_packed_attend_64(p, dtype, stream);
    if (p.a.head_dim <= 128) return launch_packed_attend_128(p, dtype, stream);
    return launch_packed_attend_256(p, dtype, stream);
}

}  // namespace specgbv
