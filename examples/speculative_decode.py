"""Speculative decoding of a batch of prompts with the library's operators: prompts and drafts go into a paged cache
(specgbv_cache_append), every model's queries attend over it (specgbv_attend_paged; the drafts of a prefix share the pages that the
prefix fills), draft tokens come from truncated distributions (specgbv_sample_filtered), the target's rows are truncated the same way, and
specgbv_verify_ex decides how many drafted tokens stay (pending_state: Algorithm 3's bookkeeping).  The models are small decoders of random
weights; their projections are plain matrix products.

`decode` keeps the block tables on the host.  `decode_on_gpu` leaves them, the positions and the texts on the GPU: pages are dealt out by
specgbv_pages_advance and positions made by specgbv_slot_map, and its caches may hold their entries in 4 bits (specgbv_packed_append,
specgbv_packed_attend).

    python examples/speculative_decode.py [--prompts 4] [--drafts 4] [--length 8] [--tokens 64] [--dtype bf16] [--on-gpu] [--packed]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2604_25925_amd as sg  # noqa: E402

DEVICE = "cuda"


class Model:
    """A decoder: per layer attention of `heads` heads in groups that share a key and value head, and a gated product."""

    def __init__(self, seed, V=2048, E=256, layers=2, heads=8, kv_heads=2, D=64, dtype=torch.bfloat16, like=None, noise=0.0):
        gen = torch.Generator(device=DEVICE).manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=gen, device=DEVICE) / math.sqrt(shape[0])).to(dtype)

        self.V, self.heads, self.kv_heads, self.D, self.dtype = V, heads, kv_heads, D, dtype
        self.inv_freq = 10000.0 ** (-torch.arange(D // 2, device=DEVICE, dtype=torch.float64) / (D // 2))
        self.embed = torch.randn((V, E), generator=gen, device=DEVICE).to(dtype)
        self.layers = [{"qkv": weight(E, (heads + 2 * kv_heads) * D), "o": weight(heads * D, E), "up": weight(E, 2 * E), "gate": weight(E, 2 * E),
                        "down": weight(2 * E, E), "q_norm": torch.ones(D, dtype=dtype, device=DEVICE),
                        "k_norm": torch.ones(D, dtype=dtype, device=DEVICE)} for _ in range(layers)]
        self.head = weight(E, V) * 3
        if like is not None:                                  # a model near to another one: what a draft model is to its target
            self.embed, self.layers = like.embed, like.layers[:layers]
            self.head = like.head + noise * weight(E, V)

    def cache(self, pages, page):
        shape = (len(self.layers), 2, pages, self.kv_heads, page, self.D)
        return torch.zeros(shape, dtype=self.dtype, device=DEVICE)

    def caches(self, pages, page, table, packed=False):
        """A cache per layer over a table of its own program."""
        if packed:
            return [sg.PackedCache.empty(pages, self.kv_heads, page, self.D, table, self.dtype) for _ in self.layers]
        return [sg.PagedCache(c[0], c[1], table) for c in self.cache(pages, page)]

    def forward(self, tokens, positions, caches, shared_len=None, rows=None):
        """Logits [S, rows, V] of the last `rows` tokens; tokens and positions [S, T] (position below 0: padding); caches: a PagedCache or
        PackedCache per layer, to which the tokens' keys and values are appended."""
        S, T = tokens.shape
        x = self.embed[tokens.long()]
        for w, cache in zip(self.layers, caches):
            qkv = (self.norm(x) @ w["qkv"]).view(S, T, -1, self.D)
            q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), dim=2)
            packed = isinstance(cache, sg.PackedCache)
            append, attend = (sg.specgbv_packed_append, sg.specgbv_packed_attend) if packed else (sg.specgbv_cache_append, sg.specgbv_attend_paged)
            q = append(cache, q, k, v, positions, inv_freq=self.inv_freq, q_weight=w["q_norm"], k_weight=w["k_norm"])
            a, _ = attend(cache, q, positions, shared_len=shared_len)
            x = x + a.reshape(S, T, -1) @ w["o"]
            y = self.norm(x)
            x = x + (torch.nn.functional.silu(y @ w["gate"]) * (y @ w["up"])) @ w["down"]
        return self.norm(x if rows is None else x[:, T - rows:]) @ self.head

    @staticmethod
    def norm(x):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + 1e-6)).to(x.dtype)


def right_aligned(rows):
    """int32 [n, longest] of lists, padded in front with -1."""
    T = max(1, max(len(r) for r in rows))
    return torch.tensor([[-1] * (T - len(r)) + list(r) for r in rows], dtype=torch.int32, device=DEVICE)


def decode(target, draft, prompts, drafts=4, length=8, new=64, page=16, temperature=0.8, top_k=0, top_p=0.95, min_p=0.0, seed=1):
    """Texts (lists of tokens, the prompts included) and the number of iterations.  A prompt that has `new` tokens is finished: it is padding in
    the iterations that others still need.

    Every draft has pages of its own; those of a page index that the prefix fills are the accepted draft's for all drafts of the prefix
    (the table says so, and shared_len).  The tokens behind the last whole page are fed again to every draft, so no page is ever copied."""
    B, K, L = len(prompts), drafts, length
    S, V = B * K, target.V
    text = [list(p) for p in prompts]
    width = (max(len(p) for p in prompts) + new + 2 * L + 2 * page) // page
    own = torch.arange(S * width, dtype=torch.int32).view(B, K, width)
    table = own.clone()
    dev_table = table.view(S, width).to(DEVICE)
    models = (target, draft)
    memory = [m.cache(S * width, page) for m in models]
    step = [[sg.PagedCache(c[0], c[1], dev_table) for c in mem] for mem in memory]

    gen = torch.Generator(device=DEVICE).manual_seed(seed)

    def filters(n):
        return {name: torch.full((n,), value, dtype=torch.int32 if name == "top_k" else torch.float32, device=DEVICE)
                for name, value in (("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p))}

    each, block = filters(S), filters(S * (L + 1))
    state = torch.zeros(sg.specgbv_pending_state_bytes(B), dtype=torch.uint8, device=DEVICE)

    # the prompts' whole pages, by draft 0 of each
    whole = [(len(t) - 1) // page for t in text]
    for b in range(B):
        table[b, :, :whole[b]] = own[b, 0, :whole[b]]
    dev_table.copy_(table.view(S, width))
    if any(whole):
        at = right_aligned([range(w * page) for w in whole])
        tokens = right_aligned([t[:w * page] for t, w in zip(text, whole)])
        first = dev_table.view(B, K, width)[:, 0].contiguous()
        for m, mem in zip(models, memory):
            m.forward(tokens.clamp(min=0), at, [sg.PagedCache(c[0], c[1], first) for c in mem], rows=1)

    iterations = 0
    while True:
        going = [len(t) - len(p) < new for t, p in zip(text, prompts)]
        if not any(going):
            return text, iterations
        # (a block reaches to its prompt's length + new + L - 2 at most, which the table holds)
        shared = torch.tensor([w * page if g else 0 for w, g in zip(whole, going)], dtype=torch.int32, device=DEVICE)
        tail = right_aligned([t[w * page:] if g else [] for t, w, g in zip(text, whole, going)]).repeat_interleave(K, dim=0).clamp(min=0)
        tail_at = right_aligned([range(w * page, len(t)) if g else [] for t, w, g in zip(text, whole, going)]).repeat_interleave(K, dim=0)
        end = tail_at[:, -1:].clone()                         # -1: finished
        drafted_at = torch.where(end < 0, end, end + 1 + torch.arange(L, dtype=torch.int32, device=DEVICE))

        # ---- the drafts: one token a step
        drafted = torch.empty((S, L), dtype=torch.int32, device=DEVICE)
        draft_rows = torch.empty((S, L, V), dtype=draft.dtype, device=DEVICE)
        for i in range(L):
            tokens, at = (tail, tail_at) if i == 0 else (drafted[:, i - 1:i], drafted_at[:, i - 1:i])
            z = draft.forward(tokens, at.contiguous(), step[1], shared, rows=1)
            u = torch.rand(S, generator=gen, device=DEVICE)
            drafted[:, i] = sg.specgbv_sample_filtered(z[:, 0], u, keep=True, kept=draft_rows[:, i], **each)[0]

        # ---- the target scores all blocks at once, and its rows are truncated as the drafts' were
        at = torch.cat((tail_at, drafted_at), dim=1)
        z = target.forward(torch.cat((tail, drafted), dim=1), at.contiguous(), step[0], shared, rows=L + 1)
        sg.specgbv_sample_filtered(z, draw=False, keep=True, kept=z, **block)

        # ---- what stays: accepted tokens and one more; pages that they fill become the prefix's
        taken, by, out, _ = sg.specgbv_verify_ex(z.view(B, K, L + 1, V), draft_rows.view(B, K, L, V), drafted.view(B, K, L), temperature, seed,
                                                 iterations, pending_state=state)
        iterations += 1
        taken, by, out = taken.tolist(), by.tolist(), out.tolist()
        for b in range(B):
            if not going[b]:
                continue
            # whole pages of tokens whose keys and values both models have: the draft model was not fed the last drafted token
            held = (len(text[b]) + min(taken[b], L - 1)) // page
            text[b] += out[b][:taken[b] + 1]
            table[b, :, whole[b]:held] = own[b, max(by[b], 0), whole[b]:held]
            whole[b] = held
        dev_table.copy_(table.view(S, width))


def of_first_drafts(cache, table):
    """The same pages for the first draft of each prefix alone."""
    if isinstance(cache, sg.PackedCache):
        return sg.PackedCache(cache.k, cache.v, cache.k_scale, cache.v_scale, table, cache.dtype)
    return sg.PagedCache(cache.k, cache.v, table)


def decode_on_gpu(target, draft, prompts, drafts=4, length=8, new=64, page=16, temperature=0.8, top_k=0, top_p=0.95, min_p=0.0, seed=1, packed=True):
    """`decode` with texts, tables and positions on the GPU; the host only looks at whether any prompt still goes on.

    have[b] tokens of a text are in both models' caches; pages that they fill are the prefix's, the accepted draft's become so, and the
    pages behind them hold room for the rest of the text and a block.  A prompt that has its tokens gives all its pages back."""
    B, K, L = len(prompts), drafts, length
    S, V, page_room = B * K, target.V, L + 3                  # (a text is at most two tokens ahead of what both models were fed)
    most = max(len(p) for p in prompts) + new + 2 * L + 2
    width = (most + page_room) // page + 2
    pages = B * (width + (K - 1) * (page_room // page + 3))
    pool = sg.PagePool.empty(B, width, pages, page_size=page, drafts=K, device=DEVICE)
    step = [m.caches(pages, page, pool.table, packed) for m in (target, draft)]

    def column(values):
        return torch.tensor(values, dtype=torch.int32, device=DEVICE)

    text = torch.zeros((B, most), dtype=torch.int64, device=DEVICE)
    for b, p in enumerate(prompts):
        text[b, :len(p)] = torch.tensor(p, device=DEVICE)
    at_start = column([len(p) for p in prompts])
    len_now, have, chosen = at_start.clone(), (at_start - 1).clamp(min=1), torch.zeros(B, dtype=torch.int32, device=DEVICE)
    going = torch.ones(B, dtype=torch.bool, device=DEVICE)
    gen = torch.Generator(device=DEVICE).manual_seed(seed)

    def filters(n):
        return {name: torch.full((n,), value, dtype=torch.int32 if name == "top_k" else torch.float32, device=DEVICE)
                for name, value in (("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p))}

    each, block = filters(S), filters(S * (L + 1))
    state = torch.zeros(sg.specgbv_pending_state_bytes(B), dtype=torch.uint8, device=DEVICE)

    def places(start, count, tokens, right=False, table=pool.table, per=K):
        return sg.specgbv_slot_map(table, start, count, tokens, page_size=page, pages=pages, drafts=per, right=right, flat=False)[0]

    # the prompts' whole pages, by draft 0 of each
    shared, served, ws = sg.specgbv_pages_advance(pool, have, room=page_room)
    first = pool.table.view(B, K, width)[:, 0]
    fed = max(len(p) - 1 for p in prompts) // page * page
    if fed:
        at = places(torch.zeros_like(shared), shared, fed, table=first, per=1)
        for m, caches in zip((target, draft), step):
            m.forward(text[:, :fed], at, [of_first_drafts(c, first) for c in caches], rows=1)

    iterations = 0
    while bool(going.any()):
        if iterations:
            shared, served, ws = sg.specgbv_pages_advance(pool, torch.where(going, have.clamp(min=1), 0), chosen=chosen, room=page_room, workspace=ws)
        tail_at = places(shared, torch.where(going, len_now - shared, 0), page + 2, right=True)
        tail = text.repeat_interleave(K, dim=0).gather(1, tail_at.clamp(min=0).long())
        drafted_at = places(len_now, going.int() * L, L)

        # ---- the drafts: one token a step
        drafted = torch.empty((S, L), dtype=torch.int32, device=DEVICE)
        draft_rows = torch.empty((S, L, V), dtype=draft.dtype, device=DEVICE)
        for i in range(L):
            tokens, at = (tail, tail_at) if i == 0 else (drafted[:, i - 1:i], drafted_at[:, i - 1:i].contiguous())
            z = draft.forward(tokens, at, step[1], shared, rows=1)
            u = torch.rand(S, generator=gen, device=DEVICE)
            drafted[:, i] = sg.specgbv_sample_filtered(z[:, 0], u, keep=True, kept=draft_rows[:, i], **each)[0]

        # ---- the target scores all blocks at once, and its rows are truncated as the drafts' were
        z = target.forward(torch.cat((tail, drafted.long()), dim=1), torch.cat((tail_at, drafted_at), dim=1), step[0], shared, rows=L + 1)
        sg.specgbv_sample_filtered(z, draw=False, keep=True, kept=z, **block)

        # ---- what stays: accepted tokens and one more
        taken, chosen, out, _ = sg.specgbv_verify_ex(z.view(B, K, L + 1, V), draft_rows.view(B, K, L, V), drafted.view(B, K, L), temperature, seed,
                                                     iterations, pending_state=state)
        iterations += 1
        i = torch.arange(L + 1, device=DEVICE)
        stays = going[:, None] & (i <= taken[:, None])
        where = torch.where(stays, len_now[:, None] + i, most - 1)                      # (the last column holds nothing)
        text.scatter_(1, where, torch.where(stays, out.long(), 0))
        have = torch.where(going, len_now + taken.clamp(max=L - 1), have)               # (the draft model was not fed a block's last token)
        len_now = torch.where(going, len_now + taken + 1, len_now)
        going = going & (len_now - at_start < new)
    sg.specgbv_pages_advance(pool, torch.zeros_like(have), workspace=ws)
    ends = len_now.tolist()
    return [row[:n] for row, n in zip(text.tolist(), ends)], iterations, pool


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--prompts", type=int, default=4)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--length", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--on-gpu", action="store_true", help="tables, positions and texts stay on the GPU")
    ap.add_argument("--packed", action="store_true", help="caches of 4 bits (implies --on-gpu)")
    a = ap.parse_args()
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    target = Model(1, dtype=dtype)
    draft = Model(2, dtype=dtype, like=target, noise=0.5)
    gen = torch.Generator().manual_seed(0)
    prompts = [torch.randint(target.V, (20 + 31 * i,), generator=gen).tolist() for i in range(a.prompts)]
    if a.on_gpu or a.packed:
        text, iterations, _ = decode_on_gpu(target, draft, prompts, a.drafts, a.length, a.tokens, packed=a.packed)
    else:
        text, iterations = decode(target, draft, prompts, a.drafts, a.length, a.tokens)
    made = sum(len(t) - len(p) for t, p in zip(text, prompts))
    print("%d tokens for %d prompts in %d iterations" % (made, a.prompts, iterations))


if __name__ == "__main__":
    main()
