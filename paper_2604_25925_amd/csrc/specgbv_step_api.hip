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

static specgbv_status check_append(const specgbv_paged_cache &c, const specgbv_append_args &a)
{
    const specgbv_status st = check_heads(c, a.tokens, a.heads, a.positions_stride);
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
    st = check_append(c, a);
    if (st != SPECGBV_OK || c.sequences == 0 || a.tokens == 0) return st;
    const size_t esz = element_bytes(c.dtype);
    AppendProblem p{};
    p.q = a.q; p.k = a.k; p.v = a.v; p.q_out = a.q_out; p.k_cache = c.k; p.v_cache = c.v;
    p.q_weight = a.q_weight; p.k_weight = a.k_weight; p.positions = a.positions; p.inv_freq = a.inv_freq;
    p.map = page_map(c);
    p.tokens_all = c.sequences * a.tokens;
    p.by_tokens = Divider::of(a.tokens);
    p.by_heads = Divider::of(a.heads + 2 * c.kv_heads);
    int width = static_cast<int>(16 / esz);                   // entries of a vector
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

static specgbv_status check_attend_args(const specgbv_paged_cache *cache, const specgbv_attend_args *args)
{
    if (!args) return fail(SPECGBV_EINVAL, "null arguments");
    const specgbv_status st = check_heads(*cache, args->tokens, args->heads, args->positions_stride);
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

static specgbv_status check_attend(const specgbv_paged_cache *cache, const specgbv_attend_args *args, bool pointers)
{
    const specgbv_status st = check_cache(cache, pointers);
    return st != SPECGBV_OK ? st : check_attend_args(cache, args);
}

static AttendPlan plan_of(const specgbv_paged_cache &c, const specgbv_attend_args &a, AttendPlan (*plan)(int, int, bool, int, int, int, int, int, int, int64_t))
{
    const bool shared = a.prefixes > 0;
    const int64_t held = static_cast<int64_t>(c.table_width) * c.page_size;
    return plan(c.sequences, shared ? c.sequences / a.prefixes : 1, shared, a.tokens, a.heads, c.kv_heads, c.head_dim, element_bytes(c.dtype), a.window,
                       a.max_len > 0 && a.max_len < held ? a.max_len : held);
}

// The launch's arguments, from a cache and a call's arguments that have passed their checks.
static specgbv_status attend_problem(const specgbv_paged_cache &c, const specgbv_attend_args &a,
                                     AttendPlan (*plan_for)(int, int, bool, int, int, int, int, int, int, int64_t),
                                     void *workspace, size_t workspace_bytes, AttendProblem &p)
{
    if (!a.q || !a.out || !a.positions || (a.prefixes > 0 && !a.shared_len)) return fail(SPECGBV_EINVAL, "null input or output pointer");
    const size_t esz = element_bytes(c.dtype);
    if (!aligned(a.q, esz) || !aligned(a.out, esz) || !aligned(a.positions, 4) || !aligned(a.shared_len, 4))
        return fail(SPECGBV_EINVAL, "pointer not aligned to its element size");
    const AttendPlan plan = plan_of(c, a, plan_for);
    if (plan.bytes > 0) {
        if (!workspace) return fail(SPECGBV_EWORKSPACE, "workspace is null (need %zu bytes)", plan.bytes);
        if (!aligned(workspace, 256)) return fail(SPECGBV_EWORKSPACE, "workspace must be 256-byte aligned");
        if (workspace_bytes < plan.bytes) return fail(SPECGBV_EWORKSPACE, "workspace has %zu bytes, need %zu", workspace_bytes, plan.bytes);
    }
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
    return SPECGBV_OK;
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
    AttendProblem p{};
    const specgbv_status ready = attend_problem(c, a, plan_attend, workspace, workspace_bytes, p);
    if (ready != SPECGBV_OK) return ready;
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

namespace specgbv {

// A cache of 4-bit entries as one of entries, for the checks and launches that look at sizes and the table alone; strides in bytes.
static specgbv_paged_cache view_of(const specgbv_packed_cache &c)
{
    specgbv_paged_cache v{};
    v.k = c.k; v.v = c.v; v.table = c.table;
    v.k_page_stride = c.k_page_stride; v.k_head_stride = c.k_head_stride; v.k_token_stride = c.k_token_stride;
    v.v_page_stride = c.v_page_stride; v.v_head_stride = c.v_head_stride; v.v_token_stride = c.v_token_stride;
    v.table_stride = c.table_stride;
    v.pages = c.pages; v.kv_heads = c.kv_heads; v.page_size = c.page_size; v.head_dim = c.head_dim;
    v.sequences = c.sequences; v.table_width = c.table_width; v.dtype = c.dtype;
    return v;
}

static specgbv_status check_packed(const specgbv_packed_cache *c, bool pointers)
{
    if (!c) return fail(SPECGBV_EINVAL, "null cache");
    specgbv_paged_cache v = view_of(*c);
    // (its strides are bytes: 16 of them are a whole unit whatever the type, as 4 entries of float32 are)
    for (int64_t *s : {&v.k_page_stride, &v.k_head_stride, &v.k_token_stride, &v.v_page_stride, &v.v_head_stride, &v.v_token_stride}) {
        if (*s >= 0 && *s % 16) return fail(SPECGBV_EUNSUPPORTED, "the cache's strides are not whole 16 bytes");
        if (*s > INT32_MAX) return fail(SPECGBV_EUNSUPPORTED, "a stride of the cache exceeds 2^31 - 1 bytes");
    }
    const specgbv_status st = check_cache(&v, pointers);
    if (st != SPECGBV_OK) return st;
    if (c->head_dim % 32) return fail(SPECGBV_EUNSUPPORTED, "head_dim=%d is not a multiple of 32", c->head_dim);
    const int64_t strides[6] = {c->k_scale_page_stride, c->k_scale_head_stride, c->k_scale_block_stride,
                                c->v_scale_page_stride, c->v_scale_head_stride, c->v_scale_block_stride};
    for (int64_t s : strides) {
        if (s < 0) return fail(SPECGBV_EINVAL, "negative stride");
        if (s % 8) return fail(SPECGBV_EUNSUPPORTED, "the strides of the scales are not whole 8 bytes");
        if (s > INT32_MAX) return fail(SPECGBV_EUNSUPPORTED, "a stride of the scales exceeds 2^31 - 1 bytes");
    }
    if (c->k_scale_block_stride > (1 << 26) || c->v_scale_block_stride > (1 << 26))
        return fail(SPECGBV_EUNSUPPORTED, "blocks of the scales lie more than 2^26 bytes apart");
    if (pointers) {
        if (!c->k_scale || !c->v_scale) return fail(SPECGBV_EINVAL, "null pointer in the cache");
        if (!aligned(c->k_scale, 8) || !aligned(c->v_scale, 8)) return fail(SPECGBV_EUNSUPPORTED, "the scales are not 8-byte aligned");
    }
    return SPECGBV_OK;
}

template <typename P> static void set_packed_strides(P &p, const specgbv_packed_cache &c)
{
    p.k_cache_stride[0] = c.k_page_stride; p.k_cache_stride[1] = c.k_token_stride; p.v_cache_stride[0] = c.v_page_stride; p.v_cache_stride[1] = c.v_token_stride;
    p.k_scale_page = c.k_scale_page_stride; p.v_scale_page = c.v_scale_page_stride;
    p.k_cache_head = static_cast<int32_t>(c.k_head_stride); p.v_cache_head = static_cast<int32_t>(c.v_head_stride);
    p.k_scale_head = static_cast<int32_t>(c.k_scale_head_stride); p.v_scale_head = static_cast<int32_t>(c.v_scale_head_stride);
    p.k_scale_block = static_cast<int32_t>(c.k_scale_block_stride); p.v_scale_block = static_cast<int32_t>(c.v_scale_block_stride);
}

static bool wide_rows(const void *p, const int64_t *stride, size_t esz)
{
    const int unit = static_cast<int>(16 / esz);
    return allowed_width(unit, p, stride, 3, esz) == unit;
}

static specgbv_status check_packed_attend(const specgbv_packed_cache *cache, const specgbv_attend_args *args, bool pointers)
{
    const specgbv_status st = check_packed(cache, pointers);
    if (st != SPECGBV_OK) return st;
    const specgbv_paged_cache v = view_of(*cache);
    return check_attend_args(&v, args);
}

// Bytes from a head's first to behind its last one, of an array of pages and rows in them.
static int64_t reach_of(const specgbv_packed_cache &c, int64_t page_stride, int64_t row_stride, int rows, int64_t row_bytes)
{
    return (c.pages - 1) * page_stride + (rows - 1) * row_stride + row_bytes;
}

}  // namespace specgbv

extern "C" {

specgbv_status specgbv_packed_append(const specgbv_packed_cache *cache, const specgbv_append_args *args, void *hip_stream)
{
    specgbv_status st = check_packed(cache, true);
    if (st != SPECGBV_OK) return st;
    if (!args) return fail(SPECGBV_EINVAL, "null arguments");
    const specgbv_paged_cache c = view_of(*cache);
    const specgbv_append_args &a = *args;
    st = check_append(c, a);
    if (st != SPECGBV_OK || c.sequences == 0 || a.tokens == 0) return st;
    for (int64_t stride : {a.q_stride[2], a.k_stride[2], a.v_stride[2], a.q_out_stride[2]})
        if (stride > INT32_MAX) return fail(SPECGBV_EUNSUPPORTED, "heads lie more than 2^31 - 1 entries apart");
    const size_t esz = element_bytes(c.dtype);
    PackedAppendProblem p{};
    p.q = a.q; p.k = a.k; p.v = a.v; p.q_out = a.q_out;
    p.k_cache = static_cast<uint8_t *>(cache->k); p.v_cache = static_cast<uint8_t *>(cache->v);
    p.k_scale = static_cast<uint8_t *>(cache->k_scale); p.v_scale = static_cast<uint8_t *>(cache->v_scale);
    p.q_weight = a.q_weight; p.k_weight = a.k_weight; p.positions = a.positions; p.inv_freq = a.inv_freq;
    p.map = page_map(c);
    p.tokens_all = c.sequences * a.tokens;
    p.by_tokens = Divider::of(a.tokens);
    for (int i = 0; i < 2; ++i) {
        p.q_stride[i] = a.q_stride[i]; p.k_stride[i] = a.k_stride[i]; p.v_stride[i] = a.v_stride[i]; p.q_out_stride[i] = a.q_out_stride[i];
    }
    set_packed_strides(p, *cache);
    p.q_head = static_cast<int32_t>(a.q_stride[2]); p.k_head = static_cast<int32_t>(a.k_stride[2]);
    p.v_head = static_cast<int32_t>(a.v_stride[2]); p.q_out_head = static_cast<int32_t>(a.q_out_stride[2]);
    p.positions_stride = a.positions_stride;
    p.eps = a.eps; p.inv_dim = 1.0f / c.head_dim;
    p.heads = a.heads; p.kv_heads = c.kv_heads; p.head_dim = c.head_dim; p.pairs = a.pairs; p.interleaved = a.interleaved != 0;
    const bool wide = a.pairs % 8 == 0 && wide_rows(a.q, a.q_stride, esz) && wide_rows(a.k, a.k_stride, esz) && wide_rows(a.v, a.v_stride, esz) &&
                      wide_rows(a.q_out, a.q_out_stride, esz) && aligned(a.q_weight, 16) && aligned(a.k_weight, 16);
    const hipError_t e = launch_packed_append(p, c.dtype == SPECGBV_BF16 ? 1 : 0, wide, static_cast<hipStream_t>(hip_stream));
    if (e == hipErrorInvalidConfiguration) return fail(SPECGBV_EUNSUPPORTED, "too many tokens for one launch (%d)", p.tokens_all);
    if (e != hipSuccess) return fail(SPECGBV_EHIP, "append kernel launch: %s", hipGetErrorString(e));
    return SPECGBV_OK;
}

specgbv_status specgbv_packed_read(const specgbv_packed_cache *cache, const specgbv_read_args *args, void *hip_stream)
{
    specgbv_status st = check_packed(cache, true);
    if (st != SPECGBV_OK) return st;
    if (!args) return fail(SPECGBV_EINVAL, "null arguments");
    const specgbv_paged_cache c = view_of(*cache);
    const specgbv_read_args &a = *args;
    st = check_heads(c, a.tokens, c.kv_heads, a.positions_stride);
    if (st != SPECGBV_OK) return st;
    for (int i = 0; i < 3; ++i)
        if (a.k_stride[i] < 0 || a.v_stride[i] < 0) return fail(SPECGBV_EINVAL, "negative stride");
    if (c.sequences == 0 || a.tokens == 0) return SPECGBV_OK;
    if (!a.k || !a.v || !a.positions) return fail(SPECGBV_EINVAL, "null input or output pointer");
    const size_t esz = element_bytes(c.dtype);
    if (!aligned(a.k, esz) || !aligned(a.v, esz) || !aligned(a.positions, 4)) return fail(SPECGBV_EINVAL, "pointer not aligned to its element size");
    if (c.kv_heads > (1 << 29)) return fail(SPECGBV_EUNSUPPORTED, "a token has more than 2^29 heads");
    if (a.k_stride[2] > INT32_MAX || a.v_stride[2] > INT32_MAX) return fail(SPECGBV_EUNSUPPORTED, "heads lie more than 2^31 - 1 entries apart");
    PackedReadProblem p{};
    p.k_cache = static_cast<const uint8_t *>(cache->k); p.v_cache = static_cast<const uint8_t *>(cache->v);
    p.k_scale = static_cast<const uint8_t *>(cache->k_scale); p.v_scale = static_cast<const uint8_t *>(cache->v_scale);
    p.k = a.k; p.v = a.v; p.positions = a.positions;
    p.map = page_map(c);
    p.tokens_all = c.sequences * a.tokens;
    p.by_tokens = Divider::of(a.tokens);
    set_packed_strides(p, *cache);
    for (int i = 0; i < 2; ++i) { p.k_stride[i] = a.k_stride[i]; p.v_stride[i] = a.v_stride[i]; }
    p.k_head = static_cast<int32_t>(a.k_stride[2]); p.v_head = static_cast<int32_t>(a.v_stride[2]);
    p.positions_stride = a.positions_stride;
    p.kv_heads = c.kv_heads; p.head_dim = c.head_dim;
    const hipError_t e = launch_packed_read(p, c.dtype == SPECGBV_BF16 ? 1 : 0, wide_rows(a.k, a.k_stride, esz) && wide_rows(a.v, a.v_stride, esz),
                                            static_cast<hipStream_t>(hip_stream));
    if (e == hipErrorInvalidConfiguration) return fail(SPECGBV_EUNSUPPORTED, "too many tokens for one launch (%d)", p.tokens_all);
    if (e != hipSuccess) return fail(SPECGBV_EHIP, "read kernel launch: %s", hipGetErrorString(e));
    return SPECGBV_OK;
}

size_t specgbv_packed_attend_workspace_bytes(const specgbv_packed_cache *cache, const specgbv_attend_args *args)
{
    if (check_packed_attend(cache, args, false) != SPECGBV_OK || cache->sequences == 0 || args->tokens == 0) return 0;
    const specgbv_packed_cache &c = *cache;
    const specgbv_attend_args &a = *args;
    return packed_attend_bytes(c.sequences, a.prefixes > 0 ? c.sequences / a.prefixes : 1, a.prefixes > 0, a.tokens, a.heads, c.kv_heads, c.head_dim,
                               element_bytes(c.dtype), a.window, static_cast<int64_t>(c.table_width) * c.page_size);
}

specgbv_status specgbv_packed_attend(const specgbv_packed_cache *cache, const specgbv_attend_args *args,
                                     void *workspace, size_t workspace_bytes, void *hip_stream)
{
    specgbv_status st = check_packed_attend(cache, args, true);
    if (st != SPECGBV_OK) return st;
    const specgbv_packed_cache &c = *cache;
    if (c.sequences == 0 || args->tokens == 0) return SPECGBV_OK;
    PackedProblem p{};
    st = attend_problem(view_of(c), *args, plan_packed_attend, workspace, workspace_bytes, p.a);
    if (st != SPECGBV_OK) return st;
    p.k_scale = static_cast<const uint8_t *>(c.k_scale); p.v_scale = static_cast<const uint8_t *>(c.v_scale);
    p.k_scale_page_stride = static_cast<int32_t>(c.k_scale_page_stride); p.k_scale_head_stride = static_cast<int32_t>(c.k_scale_head_stride);
    p.k_scale_block_stride = static_cast<int32_t>(c.k_scale_block_stride); p.v_scale_page_stride = static_cast<int32_t>(c.v_scale_page_stride);
    p.v_scale_head_stride = static_cast<int32_t>(c.v_scale_head_stride); p.v_scale_block_stride = static_cast<int32_t>(c.v_scale_block_stride);
    p.near = reach_of(c, c.k_page_stride, c.k_token_stride, c.page_size, c.head_dim / 2) <= UINT32_MAX &&
             reach_of(c, c.v_page_stride, c.v_token_stride, c.page_size, c.head_dim / 2) <= UINT32_MAX &&
             reach_of(c, c.k_scale_page_stride, c.k_scale_block_stride, c.head_dim / 32, c.page_size) <= UINT32_MAX &&
             reach_of(c, c.v_scale_page_stride, c.v_scale_block_stride, c.head_dim / 32, c.page_size) <= UINT32_MAX;
    const hipError_t e = launch_packed_attend(p, c.dtype == SPECGBV_BF16 ? 1 : 0, static_cast<hipStream_t>(hip_stream));
    if (e == hipErrorInvalidConfiguration) return fail(SPECGBV_EUNSUPPORTED, "too many queries for one launch");
    if (e != hipSuccess) return fail(SPECGBV_EHIP, "attention kernel launch: %s", hipGetErrorString(e));
    return SPECGBV_OK;
}

}  // extern "C"

namespace specgbv {

static specgbv_status check_pool(const specgbv_page_pool *p)
{
    if (!p) return fail(SPECGBV_EINVAL, "null pool");
    if (p->pages < 1 || p->page_size < 1 || p->prefixes < 0 || p->drafts < 1 || p->table_width < 1)
        return fail(SPECGBV_EINVAL, "a pool has pages, page_size, drafts, table_width >= 1 and prefixes >= 0 (got %d %d %d %d %d)",
                    p->pages, p->page_size, p->drafts, p->table_width, p->prefixes);
    if (p->pages >= 1 << 30) return fail(SPECGBV_EUNSUPPORTED, "pages=%d exceeds 2^30 - 1", p->pages);
    if (static_cast<int64_t>(p->table_width) * p->page_size > (1 << 30))
        return fail(SPECGBV_EUNSUPPORTED, "a sequence of %d pages of %d tokens is too long", p->table_width, p->page_size);
    if (static_cast<double>(p->prefixes) * p->drafts * p->table_width > 1073741824.0)
        return fail(SPECGBV_EUNSUPPORTED, "a table of more than 2^30 entries");
    if (p->table_stride < p->table_width && static_cast<int64_t>(p->prefixes) * p->drafts > 1)
        return fail(SPECGBV_EINVAL, "table_stride is less than table_width");
    return SPECGBV_OK;
}

}  // namespace specgbv

extern "C" {

size_t specgbv_pages_workspace_bytes(const specgbv_page_pool *pool)
{
    if (check_pool(pool) != SPECGBV_OK || pool->prefixes == 0) return 0;
    return pages_bytes(pool->prefixes, pool->drafts, pool->table_width);
}

specgbv_status specgbv_pages_advance(const specgbv_page_pool *pool, const specgbv_advance_args *args, void *workspace, size_t workspace_bytes,
                                     void *hip_stream)
{
    const specgbv_status st = check_pool(pool);
    if (st != SPECGBV_OK) return st;
    if (!args) return fail(SPECGBV_EINVAL, "null arguments");
    const specgbv_page_pool &c = *pool;
    const specgbv_advance_args &a = *args;
    if (a.room < 0) return fail(SPECGBV_EINVAL, "room must be >= 0 (got %d)", a.room);
    if (c.prefixes == 0) return SPECGBV_OK;
    if (!c.table || !c.ring || !c.ends || !c.held) return fail(SPECGBV_EINVAL, "null pointer in the pool");
    if (!a.length || !a.shared_len || !a.served) return fail(SPECGBV_EINVAL, "null input or output pointer");
    for (const void *p : {static_cast<const void *>(c.table), static_cast<const void *>(c.ring), static_cast<const void *>(c.ends), static_cast<const void *>(c.held),
                          static_cast<const void *>(a.length), static_cast<const void *>(a.chosen), static_cast<const void *>(a.shared_len),
                          static_cast<const void *>(a.served)})
        if (!aligned(p, 4)) return fail(SPECGBV_EINVAL, "pointer not aligned to its element size");
    const size_t need = pages_bytes(c.prefixes, c.drafts, c.table_width);
    if (need > 0) {
        if (!workspace) return fail(SPECGBV_EWORKSPACE, "workspace is null (need %zu bytes)", need);
        if (!aligned(workspace, 256)) return fail(SPECGBV_EWORKSPACE, "workspace must be 256-byte aligned");
        if (workspace_bytes < need) return fail(SPECGBV_EWORKSPACE, "workspace has %zu bytes, need %zu", workspace_bytes, need);
    }
    const PagesProblem p{c.table, c.ring, c.ends, c.held, a.length, a.chosen, a.shared_len, a.served, workspace, c.table_stride,
                         Divider::of(c.page_size), c.pages, c.prefixes, c.drafts, c.table_width, a.room};
    const hipError_t e = launch_pages(p, static_cast<hipStream_t>(hip_stream));
    if (e == hipErrorInvalidConfiguration) return fail(SPECGBV_EUNSUPPORTED, "too many prefixes for one launch (%d)", c.prefixes);
    if (e != hipSuccess) return fail(SPECGBV_EHIP, "pages kernel launch: %s", hipGetErrorString(e));
    return SPECGBV_OK;
}

specgbv_status specgbv_slot_map(const specgbv_slot_args *args, void *hip_stream)
{
    if (!args) return fail(SPECGBV_EINVAL, "null arguments");
    const specgbv_slot_args &a = *args;
    if (a.sequences < 0 || a.drafts < 1 || a.table_width < 1 || a.page_size < 1 || a.pages < 1 || a.tokens < 0)
        return fail(SPECGBV_EINVAL, "sizes must satisfy sequences, tokens >= 0, drafts, table_width, page_size, pages >= 1 (got %d %d %d %d %d %d)",
                    a.sequences, a.tokens, a.drafts, a.table_width, a.page_size, a.pages);
    if (a.sequences % a.drafts) return fail(SPECGBV_EINVAL, "%d sequences are not prefixes of %d drafts", a.sequences, a.drafts);
    if (static_cast<int64_t>(a.table_width) * a.page_size > (1 << 30))
        return fail(SPECGBV_EUNSUPPORTED, "a sequence of %d pages of %d tokens is too long", a.table_width, a.page_size);
    if (static_cast<double>(a.sequences) * a.tokens > 1.0e9) return fail(SPECGBV_EUNSUPPORTED, "too many tokens for one call");
    if (a.sequences > 1 && (a.table_stride < a.table_width || a.positions_stride < a.tokens || (a.slots && a.slots_stride < a.tokens)))
        return fail(SPECGBV_EINVAL, "rows of the table, positions or slots overlap");
    if (a.sequences == 0 || a.tokens == 0) return SPECGBV_OK;
    if (!a.start || !a.count || !a.positions || (a.slots && !a.table)) return fail(SPECGBV_EINVAL, "null input or output pointer");
    if (!aligned(a.table, 4) || !aligned(a.start, 4) || !aligned(a.count, 4) || !aligned(a.positions, 4) || !aligned(a.slots, 8))
        return fail(SPECGBV_EINVAL, "pointer not aligned to its element size");
    SlotsProblem p{};
    p.map = PageMap{a.table, a.table_stride, Divider::of(a.page_size), a.pages, a.table_width};
    p.start = a.start; p.count = a.count; p.positions = a.positions; p.slots = a.slots;
    p.positions_stride = a.positions_stride; p.slots_stride = a.slots_stride;
    p.by_tokens = Divider::of(a.tokens); p.by_drafts = Divider::of(a.drafts);
    p.sequences = a.sequences; p.tokens = a.tokens; p.right = a.right != 0;
    const hipError_t e = launch_slots(p, static_cast<hipStream_t>(hip_stream));
    if (e == hipErrorInvalidConfiguration) return fail(SPECGBV_EUNSUPPORTED, "too many tokens for one launch");
    if (e != hipSuccess) return fail(SPECGBV_EHIP, "slots kernel launch: %s", hipGetErrorString(e));
    return SPECGBV_OK;
}

}  // extern "C"
