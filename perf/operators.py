"""Cases of the operators that a decoding step around the verification needs: appending to a paged cache, attention over
it, truncated sampling.

Shapes are those of the repository's workloads (32 prefixes of K = 8 drafts of L = 8 tokens, vocabularies of 32000 to
152064 entries, bfloat16 and float32) and, for heads and caches, generic ones.  A cache holds more pages than are in use, its
pages are dealt out in random order, and the drafts of a prefix share the pages that hold the prefix.

`run` computes an operator by elementary operations, in 32 bits, where `own` is false (angles, and everything that decides
which token is kept or drawn, in 64), and by the library's entry points where it is true.  `exact` has the same from the
definitions in 64 bits, sequence by sequence and row by row.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# -------------------------------------------------------------------------------------------------------------- cases


def listed():
    return [
        # one prompt, one drafted token, a small draft model: nothing but launches and latency
        _attend("attend_one_token", 1, 1, 1, 8, 2, 64, "bf16", 200, 16, ragged=False),
        # a drafting step of the benchmark's batch: 32 prefixes of 8 drafts, one token each, prefixes of different lengths
        _attend("attend_drafting", 32, 8, 1, 32, 8, 128, "bf16", 2048, 16),
        # the target model scores blocks of 8 drafted tokens and the bonus row: 9 queries a draft
        _attend("attend_scoring", 8, 8, 9, 32, 8, 128, "bf16", 4096, 64),
        # few sequences over long contexts: the split over the length
        _attend("attend_long_context", 4, 1, 1, 32, 8, 128, "bf16", 131072, 64, ragged=False),
        # float32, odd group of heads, pages in token order, a sliding window, sequences that are still empty
        _attend("attend_window_f32", 24, 1, 5, 14, 2, 64, "f32", 2900, 32, window=1000, token_major=True),
        # one drafted token of one prompt
        _append("append_one_token", 1, 1, 8, 2, 64, "bf16", 4096, 16),
        # the drafting step above: norms of queries and keys and the rotation
        _append("append_drafting", 256, 1, 32, 8, 128, "bf16", 8192, 16, norm=True),
        # prompts of different lengths, padded to the longest
        _append("append_prompts", 5, 4001, 32, 8, 128, "bf16", 4001, 64, token_major=True),
        # one prompt's next token from the usual three filters
        _sample("sample_one_prompt", 1, 32000, "bf16", "all", head=50),
        # the draft tokens of a position, every request with filters of its own, most of them top-p
        _sample("sample_drafts", 256, 128256, "bf16", "mixed", head=200),
        # the target rows of a batch's blocks are truncated as the drafts were: logits out, no tokens
        _sample("filter_target_rows", 1152, 32000, "bf16", "top_p", draw=False, keep=True, head=50),
        # float32 rows of an odd vocabulary, tokens and the truncated rows they were drawn from
        _sample("sample_and_filter_f32", 287, 32003, "f32", "mixed", keep=True, head=50),
    ]


def _attend(name, prefixes, drafts, new, heads, kv_heads, dim, dtype, context, page, ragged=True, window=0, token_major=False):
    c = {"op": "attend", "prefixes": prefixes, "drafts": drafts, "new": new, "heads": heads, "kv_heads": kv_heads, "dim": dim,
         "dtype": dtype, "context": context, "page": page, "ragged": ragged, "window": window, "token_major": token_major}
    return dict(c, name=name) if name else c


def _append(name, sequences, new, heads, kv_heads, dim, dtype, context, page, norm=False, rotate=None, interleaved=False,
            token_major=False):
    c = {"op": "append", "sequences": sequences, "new": new, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
         "context": context, "page": page, "norm": norm, "rotate": dim if rotate is None else rotate, "interleaved": interleaved,
         "token_major": token_major}
    return dict(c, name=name) if name else c


def _sample(name, rows, vocabulary, dtype, filters, draw=True, keep=False, head=0):
    c = {"op": "sample", "rows": rows, "vocabulary": vocabulary, "dtype": dtype, "filters": filters, "draw": draw, "keep": keep,
         "head": head}
    return dict(c, name=name) if name else c


def draw(rng):
    """Sizes between the smallest and the largest listed ones, any head layout, page size and filter."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["attend", "attend", "append", "sample", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "sample":
        V = log_int(1000, 152064)
        V -= V % rng.choice([1, 1, 2, 8, 64])
        rows = min(log_int(1, 1500), max(1, 30_000_000 // V))
        keep = rng.random() < 0.4
        return _sample(None, rows, V, dtype, rng.choice(["none", "top_k", "top_p", "min_p", "all", "mixed"]),
                       draw=not keep or rng.random() < 0.5, keep=keep, head=0 if V < 2000 else rng.choice([0, 50, 200]))
    dim = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    token_major = rng.random() < 0.5
    if op == "append":
        new = rng.choice([1, 1, 5, 9, log_int(16, 4000)])
        sequences = min(log_int(1, 256), max(1, 80_000_000 // (new * (heads + 2 * kv_heads) * dim)))
        rotate = rng.choice([dim, dim, dim // 2, 0])
        return _append(None, sequences, new, heads, kv_heads, dim, dtype, new + log_int(1, 8000), page, norm=rng.random() < 0.5,
                       rotate=rotate, interleaved=rng.random() < 0.3, token_major=token_major)
    new, drafts = rng.choice([1, 1, 2, 5, 9, 17]), rng.choice([1, 1, 2, 4, 8])
    context = log_int(40, 32768)
    prefixes = log_int(1, 64)
    most = 500_000_000                               # cache entries that a plain pass gathers
    while prefixes > 1 and (prefixes * drafts * context * max(kv_heads * dim, heads * new) > most
                            or prefixes * drafts * context * new * heads * dim > 8_000_000_000):
        prefixes = (prefixes + 1) // 2
    return _attend(None, prefixes, drafts, new, heads, kv_heads, dim, dtype, context, page, ragged=rng.random() < 0.8,
                   window=rng.choice([0, 0, 0, max(1, context // 3)]), token_major=token_major)


# ------------------------------------------------------------------------------------------------------------- inputs


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed) * 1000003 + 29)
    return gen


def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32 if dtype is torch.float32 else dtype) * scale


def _cache(gen, case, pages, dtype):
    """(k, v) as [pages, kv_heads, page, dim], held in that order or with the tokens of a page before its heads."""
    H, P, D = case["kv_heads"], case["page"], case["dim"]
    shape = (pages, P, H, D) if case["token_major"] else (pages, H, P, D)
    kv = [_normal(gen, shape, dtype) for _ in range(2)]
    return [x.transpose(1, 2) if case["token_major"] else x for x in kv]


def prepare(case, seed):
    return {"attend": _prepare_attend, "append": _prepare_append, "sample": _prepare_sample}[case["op"]](case, seed)


def _prepare_attend(case, seed):
    gen, dtype = _generator(seed), DTYPES[case["dtype"]]
    B, K, T, P, context = (case[k] for k in ("prefixes", "drafts", "new", "page", "context"))
    S = B * K
    if case["ragged"]:
        length = torch.randint(0, context + 1, (B,), generator=gen, device=DEVICE)
        length[0] = context                                      # (the longest is there)
    else:
        length = torch.full((B,), context, device=DEVICE)
    after = torch.randint(0, 8, (B, 1), generator=gen, device=DEVICE) if K > 1 else 0     # tokens drafted before these
    positions = (length[:, None] + after).expand(B, K)[..., None] + torch.arange(T, device=DEVICE)
    if K == 1:
        positions = positions - T                                # the last T tokens of the context; what lies before it is not there
    positions = positions.reshape(S, T).clamp(min=-1).to(torch.int32).contiguous()
    width = (context + 8 + T + P - 1) // P                       # pages of a sequence at most
    whole = (length // P).to(torch.int32)                        # pages that the prefix fills: shared by its drafts
    used = S * width
    pages = torch.randperm(used + 7, generator=gen, device=DEVICE)[:used].to(torch.int32).reshape(B, K, width)
    shared = torch.arange(width, device=DEVICE) < whole[:, None, None]
    table = torch.where(shared, pages[:, :1], pages).reshape(S, width).contiguous()
    k, v = _cache(gen, case, used + 7, dtype) if K == 1 else _cache_of(gen, case, table, dtype)
    q = _normal(gen, (S, T, case["heads"], case["dim"]), dtype, 2.0)
    return {"case": case, "q": q, "k": k, "v": v, "table": table, "positions": positions,
            "shared_len": whole * P if K > 1 else None, "max_len": context + 8 + T}


def _cache_of(gen, case, table, dtype):
    """A cache of no more pages than the table uses: the pages that drafts share are few; the table is renumbered in place."""
    ids, place = torch.unique(table, return_inverse=True)
    order = torch.randperm(ids.numel(), generator=gen, device=DEVICE)
    table.copy_(order[place].reshape(table.shape).to(torch.int32))
    return _cache(gen, case, ids.numel(), dtype)


def _prepare_append(case, seed):
    gen, dtype = _generator(seed), DTYPES[case["dtype"]]
    S, T, H, G, D, P, context = (case[k] for k in ("sequences", "new", "heads", "kv_heads", "dim", "page", "context"))
    width = (context + P - 1) // P
    start = torch.randint(0, context - T + 1, (S, 1), generator=gen, device=DEVICE)
    step = torch.arange(T, device=DEVICE)
    count = torch.randint(T // 3 + 1, T + 1, (S, 1), generator=gen, device=DEVICE)       # padded where a prompt is shorter
    positions = torch.where(step < count, start + step, -1).to(torch.int32).contiguous()
    near = (T + 2 * P - 2) // P                                  # pages that the new tokens touch; the others are of no matter
    ids = torch.randperm(S * near + 3, generator=gen, device=DEVICE)[:S * near].to(torch.int32).reshape(S, near)
    first = (start // P).to(torch.int64)
    at = torch.arange(width, device=DEVICE) - first
    table = torch.where((at >= 0) & (at < near), ids.gather(1, at.clamp(0, near - 1)), 0).to(torch.int32).contiguous()
    k_cache, v_cache = _cache(gen, case, S * near + 3, dtype)
    qkv = _normal(gen, (S, T, H + 2 * G, D), dtype)              # the projections' output: heads of q, k and v side by side
    R = case["rotate"] // 2
    inv_freq = 10000.0 ** (-torch.arange(R, device=DEVICE, dtype=torch.float64) / max(R, 1)) if R else None
    weight = [(1.0 + 0.2 * torch.randn(D, generator=gen, device=DEVICE)).to(dtype) for _ in range(2)] if case["norm"] else [None, None]
    return {"case": case, "q": qkv[:, :, :H], "k": qkv[:, :, H:H + G], "v": qkv[:, :, H + G:], "k_cache": k_cache, "v_cache": v_cache,
            "table": table, "positions": positions, "inv_freq": inv_freq, "q_weight": weight[0], "k_weight": weight[1], "eps": 1e-6}


def _prepare_sample(case, seed):
    gen, dtype = _generator(seed), DTYPES[case["dtype"]]
    R, V, head = case["rows"], case["vocabulary"], case["head"]
    z = torch.randn((R, V), generator=gen, device=DEVICE) * 3.0
    if head:                                                     # few likely tokens, as language models have them
        boost = 6.0 - 1.1 * torch.log(torch.arange(1, head + 1, dtype=torch.float32, device=DEVICE))
        z.scatter_add_(1, torch.randint(V, (R, head), generator=gen, device=DEVICE), boost.expand(R, head))
    z[:, V - V // 100:] = -math.inf                              # places of the vocabulary that hold no token
    pick = lambda values: torch.tensor(values, device=DEVICE)[torch.randint(len(values), (R,), generator=gen, device=DEVICE)]
    f, some = case["filters"], torch.rand(R, generator=gen, device=DEVICE)
    s = {"case": case, "logits": z.to(dtype), "temperature": pick([0.4, 0.7, 0.8, 1.0, 1.0]).float(), "top_k": None, "top_p": None,
         "min_p": None, "u": torch.rand(R, generator=gen, device=DEVICE)}
    if f in ("top_k", "all", "mixed"):
        s["top_k"] = pick([20, 50, 50, 200, 1000]).to(torch.int32)
    if f in ("top_p", "all", "mixed"):
        s["top_p"] = pick([0.8, 0.9, 0.95, 0.99]).float()
    if f in ("min_p", "all", "mixed"):
        s["min_p"] = pick([0.01, 0.05, 0.1]).float()
    if f == "mixed":                                             # every request has its own: most use top-p alone
        s["top_k"] = torch.where(some < 0.25, s["top_k"], 0)
        s["min_p"] = torch.where(some > 0.85, s["min_p"], 0.0)
        s["top_p"] = torch.where((some > 0.2) & (some < 0.9), s["top_p"], 1.0)
    return s


# ---------------------------------------------------------------------------------------------------------------- run


def run(s):
    op = s["case"]["op"]
    if own:
        return {"attend": _own_attend, "append": _own_append, "sample": _own_sample}[op](s)
    return {"attend": _plain_attend, "append": _plain_append, "sample": _plain_sample}[op](s)


def _own_attend(s):
    """The handle of the cache, the workspace and the output are kept between the steps of a decoding loop."""
    import paper_2604_25925_amd as sg
    if "handle" not in s:
        s["handle"] = sg.PagedCache(s["k"], s["v"], s["table"])
        s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
        s["workspace"] = None
    s["out"], s["workspace"] = sg.specgbv_attend_paged(s["handle"], s["q"], s["positions"], window=s["case"]["window"],
                                                       shared_len=s["shared_len"], max_len=s["max_len"], out=s["out"],
                                                       workspace=s["workspace"])
    return {"out": s["out"]}


def _own_append(s):
    import paper_2604_25925_amd as sg
    if "handle" not in s:
        s["handle"] = sg.PagedCache(s["k_cache"], s["v_cache"], s["table"])
        s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
    sg.specgbv_cache_append(s["handle"], s["q"], s["k"], s["v"], s["positions"], inv_freq=s["inv_freq"],
                            interleaved=s["case"]["interleaved"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"],
                            out=s["out"])
    return {"q": s["out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_sample(s):
    import paper_2604_25925_amd as sg
    c = s["case"]
    if "workspace" not in s:
        s["workspace"] = None
        s["out"] = torch.empty(c["rows"], dtype=torch.int32, device=DEVICE) if c["draw"] else None
        s["kept"] = torch.empty_like(s["logits"]) if c["keep"] else None
    tokens, kept, s["workspace"] = sg.specgbv_sample_filtered(
        s["logits"], s["u"] if c["draw"] else None, temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
        draw=c["draw"], keep=c["keep"], out=s["out"], kept=s["kept"], workspace=s["workspace"])
    return {n: x for n, x in (("tokens", tokens), ("kept", kept)) if x is not None}


def _plain_attend(s):
    c, q, pos = s["case"], s["q"], s["positions"].long()
    S, T, H, D = q.shape
    G, P = c["kv_heads"], c["page"]
    width = s["table"].shape[1]
    pages = s["table"].long()
    k = s["k"][pages].float().transpose(2, 3).reshape(S, width * P, G, D).transpose(1, 2).contiguous()     # [S, G, keys, D]
    v = s["v"][pages].float().transpose(2, 3).reshape(S, width * P, G, D).transpose(1, 2).contiguous()
    rows = q.float().reshape(S, T, G, H // G, D).permute(0, 2, 1, 3, 4).reshape(S, G, T * (H // G), D).contiguous()
    score = torch.matmul(rows, k.transpose(2, 3).contiguous()) / math.sqrt(D)
    at = torch.arange(width * P, device=q.device)
    seen = (at <= pos[..., None]) & ((at > pos[..., None] - c["window"]) if c["window"] else True)         # [S, T, keys]
    seen = seen[:, None, :, None].expand(S, 1, T, H // G, width * P).reshape(S, 1, T * (H // G), width * P)
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(dim=-1, keepdim=True).clamp(min=-3.0e38)
    w = torch.exp(score - top)
    total = w.sum(dim=-1, keepdim=True)
    out = torch.matmul(w, v) / torch.where(total > 0, total, 1.0)
    return {"out": out.reshape(S, G, T, H // G, D).permute(0, 2, 1, 3, 4).reshape(S, T, H, D).to(q.dtype)}


def _plain_append(s):
    c, pos, P = s["case"], s["positions"].long(), s["case"]["page"]
    there = pos >= 0

    def turned(x, weight):
        y = x.float()
        if weight is not None:
            y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + s["eps"]) * weight.float()
        R = c["rotate"] // 2
        if R:
            angle = pos.double()[..., None] * s["inv_freq"]                      # [S, T, R]
            cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
            a, b = (y[..., 0:2 * R:2], y[..., 1:2 * R:2]) if c["interleaved"] else (y[..., :R], y[..., R:2 * R])
            pair = (a * cos - b * sin, b * cos + a * sin)
            first = torch.stack(pair, dim=-1).flatten(-2) if c["interleaved"] else torch.cat(pair, dim=-1)
            y = torch.cat((first, y[..., 2 * R:]), dim=-1)
        return y.to(x.dtype)

    q, k = turned(s["q"], s["q_weight"]), turned(s["k"], s["k_weight"])
    page = s["table"].long().gather(1, (pos // P).clamp(min=0))
    s["k_cache"][page[there], :, (pos % P)[there]] = k[there]
    s["v_cache"][page[there], :, (pos % P)[there]] = s["v"][there]
    return {"q": q * there[:, :, None, None].to(q.dtype), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_sample(s):
    c, z = s["case"], s["logits"].float()
    V = z.shape[1]
    z, at = torch.sort(z, dim=1, descending=True, stable=True)                   # ties: the lowest index first
    w = torch.exp((z.double() - z[:, :1].double()) / s["temperature"].double()[:, None])
    keep = z > -math.inf
    if s["top_k"] is not None:
        k = torch.where(s["top_k"] > 0, s["top_k"], V)
        keep &= torch.arange(V, device=z.device) < k[:, None]
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    w = torch.where(keep, w, 0.0)
    if s["top_p"] is not None:
        run_sum = torch.cumsum(w, dim=1)
        p = torch.where(s["top_p"] < 1.0, s["top_p"].double(), 2.0)
        keep &= run_sum - w < p[:, None] * run_sum[:, -1:]
        w = torch.where(keep, w, 0.0)
    out = {}
    if c["draw"]:
        run_sum = torch.cumsum(w, dim=1)
        place = (run_sum <= s["u"].double()[:, None] * run_sum[:, -1:]).sum(dim=1, keepdim=True)
        place = torch.minimum(place, keep.sum(dim=1, keepdim=True) - 1)
        out["tokens"] = at.gather(1, place).squeeze(1).to(torch.int32)
    if c["keep"]:
        out["kept"] = torch.full_like(s["logits"], -math.inf).scatter_(1, at, torch.where(keep, z, -math.inf).to(s["logits"].dtype))
    return out


# --------------------------------------------------------------------------------------------------------------- work


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "sample":
        n = case["rows"] * case["vocabulary"]
        return {"bytes": n * e * (2 if case["keep"] else 1) + case["rows"] * 20, "flops": 12 * n}
    H, G, D, T = case["heads"], case["kv_heads"], case["dim"], case["new"]
    if case["op"] == "append":
        tokens = case["sequences"] * (T if T < 3 else 0.67 * T)                  # the others are padding
        return {"bytes": int(tokens * (2 * H + 4 * G) * D * e), "flops": int(10 * tokens * (H + G) * D)}
    S, seen = case["prefixes"] * case["drafts"], case["context"]
    if case["window"]:
        seen = min(seen, case["window"])
    if case["ragged"]:
        seen *= 0.5
    kept = case["prefixes"] * seen + (S * (4 + T + case["page"] / 2) if case["drafts"] > 1 else 0)
    return {"bytes": int(2 * S * T * H * D * e + 2 * kept * G * D * e), "flops": int(4 * S * T * H * D * seen)}


# -------------------------------------------------------------------------------------------------------- in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "append": _exact_append, "sample": _exact_sample}[case["op"]](case, s)


def _exact_attend(case, s):
    """Sequence by sequence, query by query: the keys that a query sees are cut out of the cache."""
    q, positions = s["q"].double(), s["positions"].tolist()
    H, G, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE)
    for i, row in enumerate(positions):
        n = max(row) + 1
        if n <= 0:
            continue
        pages = s["table"][i, :(n + P - 1) // P].long()
        k, v = (s[x][pages].transpose(0, 1).reshape(G, -1, D)[:, :n].double() for x in ("k", "v"))
        for t, p in enumerate(row):
            if p < 0:
                continue
            lo = max(0, p + 1 - case["window"]) if case["window"] else 0
            x = q[i, t].reshape(G, H // G, D) * D ** -0.5
            a = torch.softmax(torch.bmm(x, k[:, lo:p + 1].transpose(1, 2).contiguous()), dim=-1)
            out[i, t] = torch.bmm(a, v[:, lo:p + 1].contiguous()).reshape(H, D)
    return {"out": out}


def _exact_append(case, s):
    """The rotation as a product of complex numbers."""
    P, R, pos = case["page"], case["rotate"] // 2, s["positions"]
    there = (pos >= 0).nonzero()
    where = pos[there[:, 0], there[:, 1]].long()
    page, slot = s["table"][there[:, 0], where // P].long(), where % P

    def turned(x, weight):
        y = x[there[:, 0], there[:, 1]].double()
        if weight is not None:
            y = y / torch.sqrt(torch.linalg.vector_norm(y, dim=-1, keepdim=True) ** 2 / case["dim"] + s["eps"]) * weight.double()
        if R:
            z = y[..., :2 * R]
            z = z.unflatten(-1, (R, 2)) if case["interleaved"] else z.unflatten(-1, (2, R)).transpose(-1, -2)
            turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), where[:, None].double() * s["inv_freq"])
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn[:, None])
            y[..., :2 * R] = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return y

    q = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    q[there[:, 0], there[:, 1]] = turned(s["q"], s["q_weight"])
    k, v = s["k_cache"].double(), s["v_cache"].double()
    k[page, :, slot] = turned(s["k"], s["k_weight"])
    v[page, :, slot] = s["v"][there[:, 0], there[:, 1]].double()
    return {"q": q, "k_cache": k, "v_cache": v}


def _exact_sample(case, s):
    """Row by row: the kept tokens are cut off the front of the row's order."""
    R, V = s["logits"].shape
    tokens = torch.empty(R, dtype=torch.int32, device=DEVICE)
    kept = torch.full((R, V), -math.inf, dtype=torch.float64, device=DEVICE)
    value = lambda name, r: None if s[name] is None else float(s[name][r])
    for r in range(R):
        z = s["logits"][r].double()
        order = torch.argsort(z, descending=True, stable=True)
        order = order[:int((z > -math.inf).sum())]
        k, m, p = value("top_k", r), value("min_p", r), value("top_p", r)
        if k:
            order = order[:int(k)]
        w = torch.exp((z[order] - z[order[0]]) / float(s["temperature"][r]))
        if m is not None:
            w = w[:int((w >= m).sum())]
        if p is not None and p < 1.0:
            w = w[:int(torch.searchsorted(torch.cumsum(w, 0), p * w.sum())) + 1]
        order = order[:w.numel()]
        if case["draw"]:
            i = int(torch.searchsorted(torch.cumsum(w, 0), float(s["u"][r]) * w.sum(), right=True))
            tokens[r] = order[min(i, w.numel() - 1)].to(torch.int32)
        kept[r, order] = z[order]
    return {n: x for n, x, wanted in (("tokens", tokens, case["draw"]), ("kept", kept, case["keep"])) if wanted}
