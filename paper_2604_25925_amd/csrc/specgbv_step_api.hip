// C ABI of the decoding step around the verification: argument checks and launches of the paged cache's and the sampler's calls.
#include <cmath>

#include "specgbv_internal.hpp"

namespace specgbv {

static size_t element_bytes(int dtype) { return dtype == SPECGBV_BF16 ? 2 : 4; }

static bool aligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// What a cache's description says by itself; `pointers`: its addresses are looked at too.
static specgbv_status check_cache(const specgbv_paged_cache *c, bool pointers)
{
    if (!c) return fail(SPECGBV_EINVAL, "null cache");
    if (c->dtype != SPECGBV_F32 && c->dtype != SPECGBV_BF16) return fail(SPECGBV_EINVAL, "unknown dtype %d", c->dtype);
    if (c->pages < 1 || c->kv_heads < 1 || c->page_size < 1 || c->head_dim < 1 || c->sequences < 0 || c->table_width < 1)
        return fail(SPECGBV_EINVAL, "a cache has pages, kv_heads, page_size, head_dim, table_width >= 1 and sequences >= 0 (got %d %d %d %d %d %d)",
                    c->pages, c->kv_heads, c->page_size, c->head_dim, c->table_width, c->sequences);
    if (c->head_dim % 8 || c->head_dim > 256)
        return fail(SPECGBV_EUNSUPPORTED, "head_dim=%d is not a multiple of 8 up to 256", c->head_dim);
    if (c->page_size % 8) return fail(SPECGBV_EUNSUPPORTED, "page_size=%d is not a multiple of 8", c->page_size);
    if (static_cast<int64_t>(c->table_width) * c->page_size > (1 << 30))
        return fail(SPECGBV_EUNSUPPORTED, "a sequence of %d pages of %d tokens is too long", c->table_width, c->page_size);
    if (c->table_stride < c->table_width && c->sequences > 1) return fail(SPECGBV_EINVAL, "table_stride is less than table_width");
    const int64_t strides[6] = {c->k_page_stride, c->k_head_stride, c->k_token_stride, c->v_page_stride, c->v_head_stride, c->v_token_stride};
    const int64_t unit = static_cast<int64_t>(16 / element_bytes(c->dtype));
    for (int64_t s : strides) {
        if (s < 0) return fail(SPECGBV_EINVAL, "negative stride");
        if (s % unit) return fail(SPECGBV_EUNSUPPORTED, "the cache's strides are not whole 16 bytes");
        if (s > INT32_MAX) return fail(SPECGBV_EUNSUPPORTED, "a stride of the cache exceeds 2^31 - 1 entries");
    }
    if (c->k_token_stride > (1 << 26) || c->v_token_stride > (1 << 26))
        return fail(SPECGBV_EUNSUPPORTED, "tokens of the cache lie more than 2^26 entries apart");
    if (pointers) {
        if (!c->k || !c->v || (!c->table && c->sequences > 0)) return fail(SPECGBV_EINVAL, "null pointer in the cache");
        if (!aligned(c->k, 16) || !aligned(c->v, 16)) return fail(SPECGBV_EUNSUPPORTED, "the cache is not 16-byte aligned");
        if (!aligned(c->table, 4)) return fail(SPECGBV_EINVAL, "pointer not aligned to its element size");
    }
    return SPECGBV_OK;
}

static PageMap page_map(const specgbv_paged_cache &c)
{
    return {c.table, c.table_stride, Divider::of(c.page_size), c.pages, c.table_width};
}

static specgbv_status check_heads(const specgbv_paged_cache &c, int tokens, int heads, int64_t positions_stride)
{
    if (tokens < 0 || heads < 1) return fail(SPECGBV_EINVAL, "sizes must satisfy tokens >= 0, heads >= 1 (got %d, %d)", tokens, heads);
    if (heads % c.kv_heads) return fail(SPECGBV_EINVAL, "heads=%d is not a multiple of kv_heads=%d", heads, c.kv_heads);
    if (positions_stride < tokens && c.sequences > 1) return fail(SPECGBV_EINVAL, "positions_stride is less than tokens");
    if (static_cast<double>(c.sequences) * tokens * heads > 1.0e9) return fail(SPECGBV_EUNSUPPORTED, "too many heads for one call");
    return SPECGBV_OK;
}

// The largest power of two of entries, at most `width`, that divides the strides and whose bytes divide the address.
static int allowed_width(int width, const void *p, const int64_t *stride, int count, size_t esz)
{
    for (; width > 1; width >>= 1) {
        bool ok = aligned(p, esz * width);
        for (int i = 0; i < count; ++i) ok = ok && stride[i] % width == 0;
        if (ok) break;
    }
    return width;
}

}  // namespace specgbv

using namespace specgbv;

extern "C" {

specgbv_status specgbv_cache_append(const specgbv_paged_cache *cache, const specgbv_append_args *args, void *hip_stream)
{
    specgbv_status st = check_cache(cache, true);
    if (st != SPECGBV_OK) return st;
    if (!args) return fail(SPECGBV_EINVAL, "null arguments");
    const specgbv_paged_cache &c = *cache;
    const specgbv_append_args &a = *args;
    st = check_heads(c, a.tokens, a.heads, a.positions_stride);
    if (st != SPECGBV_OK) return st;
    if (a.pairs < 0 || 2 * static_cast<int64_t>(a.pairs) > c.head_dim)
        return fail(SPECGBV_EINVAL, "pairs=%d does not lie in [0, head_dim / 2]", a.pairs);
    if (!(a.eps >= 0.0) || !std::isfinite(a.eps)) return fail(SPECGBV_EINVAL, "eps must be finite and >= 0 (got %g)", a.eps);
    for (int i = 0; i < 3; ++i)
        if (a.q_stride[i] < 0 || a.k_stride[i] < 0 || a.v_stride[i] < 0 || a.q_out_stride[i] < 0) return fail(SPECGBV_EINVAL, "negative stride");
    if (a.heads + 2 * static_cast<int64_t>(c.kv_heads) > (1 << 29)) return fail(SPECGBV_EUNSUPPORTED, "a token has more than 2^29 heads");
    if (c.sequences == 0 || a.tokens == 0) return SPECGBV_OK;
    if (!a.q || !a.k || !a.v || !a.q_out || !a.positions || (a.pairs > 0 && !a.inv_freq)) return fail(SPECGBV_EINVAL, "null input or output pointer");
    const size_t esz = element_bytes(c.dtype);
    if (!aligned(a.q, esz) || !aligned(a.k, esz) || !aligned(a.v, esz) || !aligned(a.q_out, esz) || !aligned(a.q_weight, esz) ||
        !aligned(a.k_weight, esz) || !aligned(a.positions, 4) || !aligned(a.inv_freq, 8))
        return fail(SPECGBV_EINVAL, "pointer not aligned to its element size");

    AppendProblem p{};
    p.q = a.q; p.k = a.k; p.v = a.v; p.q_out = a.q_out; p.k_cache = c.k; p.v_cache = c.v;
    p.q_weight = a.q_weight; p.k_weight = a.k_weight; p.positions = a.positions; p.inv_freq = a.inv_freq;
    p.map = page_map(c);
    p.tokens_all = c.sequences * a.tokens;
    p.by_tokens = Divider::of(a.tokens);
    p.by_heads = Divider::of(a.heads + 2 * c.kv_heads);
    int width = static_cast<int>(16 / esz);
    while (a.pairs % width || c.head_dim % (2 * width)) width >>= 1;
    width = allowed_width(width, a.q, a.q_stride, 3, esz);
    width = allowed_width(width, a.k, a.k_stride, 3, esz);
    width = allowed_width(width, a.v, a.v_stride, 3, esz);
    width = allowed_width(width, a.q_out, a.q_out_stride, 3, esz);
    width = allowed_width(width, a.q_weight, nullptr, 0, esz);
    width = allowed_width(width, a.k_weight, nullptr, 0, esz);
    for (int i = 0; i < 3; ++i) {
        p.q_stride[i] = a.q_stride[i]; p.k_stride[i] = a.k_stride[i]; p.v_stride[i] = a.v_stride[i]; p.q_out_stride[i] = a.q_out_stride[i];
    }
    p.k_cache_stride[0] = c.k_page_stride; p.k_cache_stride[1] = c.k_head_stride; p.k_cache_stride[2] = c.k_token_stride;
    p.v_cache_stride[0] = c.v_page_stride; p.v_cache_stride[1] = c.v_head_stride; p.v_cache_stride[2] = c.v_token_stride;
    p.positions_stride = a.positions_stride;
    p.eps = static_cast<float>(a.eps); p.inv_dim = 1.0f / c.head_dim;
    p.heads = a.heads; p.kv_heads = c.kv_heads; p.head_dim = c.head_dim; p.pairs = a.pairs; p.interleaved = a.interleaved != 0;
    const hipError_t e = launch_append(p, c.dtype == SPECGBV_BF16 ? 1 : 0, width, static_cast<hipStream_t>(hip_stream));
    if (e == hipErrorInvalidConfiguration) return fail(SPECGBV_EUNSUPPORTED, "too many tokens for one launch (%d)", p.tokens_all);
    if (e != hipSuccess) return fail(SPECGBV_EHIP, "append kernel launch: %s", hipGetErrorString(e));
    return SPECGBV_OK;
}

}  // extern "C"

namespace specgbv {

static specgbv_status check_attend(const specgbv_paged_cache *cache, const specgbv_attend_args *args, bool pointers)
{
    specgbv_status st = check_cache(cache, pointers);
    if (st != SPECGBV_OK) return st;
    if (!args) return fail(SPECGBV_EINVAL, "null arguments");
    st = check_heads(*cache, args->tokens, args->heads, args->positions_stride);
    if (st != SPECGBV_OK) return st;
    if (args->window < 0) return fail(SPECGBV_EINVAL, "window must be >= 0 (got %d)", args->window);
    if (args->max_len < 0) return fail(SPECGBV_EINVAL, "max_len must be >= 0 (got %d)", args->max_len);
    if (!(args->scale >= 0.0f) || !std::isfinite(args->scale)) return fail(SPECGBV_EINVAL, "scale must be finite and >= 0 (got %g)", (double)args->scale);
    if (args->prefixes < 0 || (args->prefixes > 0 && cache->sequences % args->prefixes))
        return fail(SPECGBV_EINVAL, "%d sequences are not drafts of %d prefixes", cache->sequences, args->prefixes);
    for (int i = 0; i < 3; ++i)
        if (args->q_stride[i] < 0 || args->out_stride[i] < 0) return fail(SPECGBV_EINVAL, "negative stride");
    return SPECGBV_OK;
}

static AttendPlan plan_of(const specgbv_paged_cache &c, const specgbv_attend_args &a)
{
    const bool shared = a.prefixes > 0;
    const int64_t held = static_cast<int64_t>(c.table_width) * c.page_size;
    return plan_attend(c.sequences, shared ? c.sequences / a.prefixes : 1, shared, a.tokens, a.heads, c.kv_heads, c.head_dim, element_bytes(c.dtype), a.window,
                       a.max_len > 0 && a.max_len < held ? a.max_len : held);
}

}  // namespace specgbv

extern "C" {

size_t specgbv_attend_workspace_bytes(const specgbv_paged_cache *cache, const specgbv_attend_args *args)
{
    if (check_attend(cache, args, false) != SPECGBV_OK || cache->sequences == 0 || args->tokens == 0) return 0;
    const specgbv_paged_cache &c = *cache;
    const specgbv_attend_args &a = *args;
    return attend_bytes(c.sequences, a.prefixes > 0 ? c.sequences / a.prefixes : 1, a.prefixes > 0, a.tokens, a.heads, c.kv_heads, c.head_dim,
                        element_bytes(c.dtype), a.window, static_cast<int64_t>(c.table_width) * c.page_size);
}

specgbv_status specgbv_attend_paged(const specgbv_paged_cache *cache, const specgbv_attend_args *args,
                                    void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const specgbv_status st = check_attend(cache, args, true);
    if (st != SPECGBV_OK) return st;
    const specgbv_paged_cache &c = *cache;
    const specgbv_attend_args &a = *args;
    if (c.sequences == 0 || a.tokens == 0) return SPECGBV_OK;
    if (!a.q || !a.out || !a.positions || (a.prefixes > 0 && !a.shared_len)) return fail(SPECGBV_EINVAL, "null input or output pointer");
    const size_t esz = element_bytes(c.dtype);
    if (!aligned(a.q, esz) || !aligned(a.out, esz) || !aligned(a.positions, 4) || !aligned(a.shared_len, 4))
        return fail(SPECGBV_EINVAL, "pointer not aligned to its element size");
    const AttendPlan plan = plan_of(c, a);
    if (plan.bytes > 0) {
        if (!workspace) return fail(SPECGBV_EWORKSPACE, "workspace is null (need %zu bytes)", plan.bytes);
        if (!aligned(workspace, 256)) return fail(SPECGBV_EWORKSPACE, "workspace must be 256-byte aligned");
        if (workspace_bytes < plan.bytes) return fail(SPECGBV_EWORKSPACE, "workspace has %zu bytes, need %zu", workspace_bytes, plan.bytes);
    }
    AttendProblem p{};
    p.q = a.q; p.k = c.k; p.v = c.v; p.out = a.out; p.positions = a.positions;
    p.shared_len = plan.shared ? a.shared_len : nullptr;
    p.map = page_map(c);
    for (int i = 0; i < 3; ++i) { p.q_stride[i] = a.q_stride[i]; p.out_stride[i] = a.out_stride[i]; }
    p.positions_stride = a.positions_stride;
    p.k_page_stride = static_cast<int32_t>(c.k_page_stride); p.k_head_stride = static_cast<int32_t>(c.k_head_stride);
    p.k_token_stride = static_cast<int32_t>(c.k_token_stride); p.v_page_stride = static_cast<int32_t>(c.v_page_stride);
    p.v_head_stride = static_cast<int32_t>(c.v_head_stride); p.v_token_stride = static_cast<int32_t>(c.v_token_stride);
    if (plan.ml_bytes > 0) {
        char *ws = static_cast<char *>(workspace);
        p.places = reinterpret_cast<int2 *>(ws);
        p.ml = reinterpret_cast<float2 *>(ws + plan.places_bytes);
        p.acc = reinterpret_cast<float *>(ws + plan.places_bytes + plan.ml_bytes);
    }
    p.c = static_cast<float>((a.scale > 0.0f ? static_cast<double>(a.scale) : 1.0 / std::sqrt(static_cast<double>(c.head_dim))) * 1.4426950408889634074);
    p.sequences = c.sequences; p.tokens = a.tokens; p.heads = a.heads; p.kv_heads = c.kv_heads; p.group = a.heads / c.kv_heads;
    p.head_dim = c.head_dim; p.drafts = plan.drafts; p.few = plan.few; p.lone = plan.lone; p.window = a.window;
    p.units = plan.units; p.all_parts = plan.all_parts; p.balanced = plan.balanced; p.most_parts = plan.most_parts;
    p.own_keys = plan.own_keys; p.grain = plan.grain; p.chunks = plan.chunks; p.chunk_keys = plan.chunk_keys;
    p.block_rows = plan.block_rows; p.row_blocks = plan.row_blocks;
    p.by_kv_heads = Divider::of(p.kv_heads);
    p.by_chunks = Divider::of(plan.chunks > 0 ? plan.chunks : 1);
    p.by_in_draft = Divider::of(p.tokens * p.group);
    p.by_group = Divider::of(p.group);
    p.by_rows = Divider::of(p.tokens * p.group * p.drafts);
    const int unit = static_cast<int>(16 / esz);
    p.q_wide = allowed_width(unit, a.q, a.q_stride, 3, esz) == unit;
    p.out_wide = allowed_width(unit, a.out, a.out_stride, 3, esz) == unit;
    const hipError_t e = launch_attend(p, c.dtype == SPECGBV_BF16 ? 1 : 0, static_cast<hipStream_t>(hip_stream));
    if (e == hipErrorInvalidConfiguration) return fail(SPECGBV_EUNSUPPORTED, "too many queries for one launch");
    if (e != hipSuccess) return fail(SPECGBV_EHIP, "attention kernel launch: %s", hipGetErrorString(e));
    return SPECGBV_OK;
}

}  // extern "C"

extern "C" {

size_t specgbv_filter_workspace_bytes(int rows, int V, specgbv_dtype dtype)
{
    (void)rows; (void)V; (void)dtype;
    return 0;
}

specgbv_status specgbv_sample_filtered(
    const void *logits, int64_t row_stride, int rows, int V, specgbv_dtype dtype,
    const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p, const float *u,
    int32_t *out_tokens, void *kept, int64_t kept_stride,
    void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (rows < 0 || V < 1) return fail(SPECGBV_EINVAL, "sizes must satisfy rows >= 0, V >= 1 (got rows=%d V=%d)", rows, V);
    if (dtype != SPECGBV_F32 && dtype != SPECGBV_BF16) return fail(SPECGBV_EINVAL, "unknown dtype %d", (int)dtype);
    if (V > (1 << 20)) return fail(SPECGBV_EUNSUPPORTED, "V=%d exceeds 1048576", V);
    if (rows >= 1 << 22) return fail(SPECGBV_EUNSUPPORTED, "rows=%d exceeds 2^22 - 1", rows);
    if (rows == 0) return SPECGBV_OK;
    if (!logits || (!out_tokens && !kept) || (out_tokens && !u)) return fail(SPECGBV_EINVAL, "null input or output pointer");
    if (rows > 1 && (row_stride < V || (kept && kept_stride < V))) return fail(SPECGBV_EINVAL, "a row stride is less than V=%d", V);
    const size_t esz = element_bytes(dtype);
    if (!aligned(logits, esz) || !aligned(kept, esz) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) ||
        !aligned(min_p, 4) || !aligned(u, 4) || !aligned(out_tokens, 4))
        return fail(SPECGBV_EINVAL, "pointer not aligned to its element size");
    (void)workspace; (void)workspace_bytes;                   // (none is needed)
    const FilterProblem p{logits, kept, row_stride, kept_stride, temperature, top_p, min_p, u, top_k, out_tokens, rows, V};
    const hipError_t e = launch_filter(p, dtype == SPECGBV_BF16 ? 1 : 0, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return fail(SPECGBV_EHIP, "filter kernel launch: %s", hipGetErrorString(e));
    return SPECGBV_OK;
}

}  // extern "C"
