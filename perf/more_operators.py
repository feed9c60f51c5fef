"""Cases of the operators around a paged cache held in 4 bits: appending to it, attention over it, block tables dealt out to
requests and their drafts, and the places of new tokens.

A cache holds every entry of a key or value in 4 bits (one sign, two exponent, one mantissa bit: 0, 1/2, 1, 3/2, 2, 3, 4, 6) and one power of
two for each 32 entries of a head.  Shapes are those of the repository's workloads (32 prefixes of K = 8 drafts of L = 8 tokens, and
bfloat16 and float32 throughout) and, for heads, pages and lengths, generic ones.

`run` computes an operator by elementary operations, in 32 bits, where `own` is false (what decides which 4-bit value an entry gets, in 64:
most entries lie next to no border, but there are millions), and by the library's entry points where it is true.  `exact` has the same from
the definitions in 64 bits.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 32                                           # entries that share a power of two


# -------------------------------------------------------------------------------------------------------------- cases


def listed():
    return [
        # one prompt, one drafted token, a small draft model: nothing but launches and latency
        _attend("attend4_one_token", 1, 1, 1, 8, 2, 64, "bf16", 200, 16, ragged=False),
        # a drafting step of the benchmark's batch: 32 prefixes of 8 drafts, one token each, prefixes of different lengths
        _attend("attend4_drafting", 32, 8, 1, 32, 8, 128, "bf16", 2048, 16),
        # the target model scores blocks of 8 drafted tokens and the bonus row: 9 queries a draft
        _attend("attend4_scoring", 8, 8, 9, 32, 8, 128, "bf16", 4096, 64),
        # few sequences over long contexts, where a cache of 4 bits counts most
        _attend("attend4_long_context", 4, 1, 1, 32, 8, 128, "bf16", 131072, 64, ragged=False),
        # float32, odd group of heads, pages in token order, a sliding window, sequences that are still empty
        _attend("attend4_window_f32", 24, 1, 5, 14, 2, 64, "f32", 2900, 32, window=1000, token_major=True),
        # one drafted token of one prompt
        _append("append4_one_token", 1, 1, 8, 2, 64, "bf16", 4096, 16),
        # the drafting step above: norms of queries and keys and the rotation
        _append("append4_drafting", 256, 1, 32, 8, 128, "bf16", 8192, 16, norm=True),
        # prompts of different lengths, padded to the longest
        _append("append4_prompts", 5, 4001, 32, 8, 128, "bf16", 4001, 64, token_major=True),
        # pages of the benchmark's batch after a verification
        _pages("pages_drafting", 32, 8, 2048, 16),
        # a large batch of requests with few drafts, and not enough pages for all of them
        _pages("pages_large_batch", 1000, 4, 8192, 16, tight=True),
        # where the next block's tokens lie, for that batch
        _slots("slots_drafting", 32, 8, 24, 2048, 16),
        # prompts of different lengths
        _slots("slots_prompts", 64, 1, 4001, 4001, 64, right=False),
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


def _pages(name, prefixes, drafts, context, page, room=17, tight=False):
    c = {"op": "pages", "prefixes": prefixes, "drafts": drafts, "context": context, "page": page, "room": room, "tight": tight}
    return dict(c, name=name) if name else c


def _slots(name, prefixes, drafts, tokens, context, page, right=True):
    c = {"op": "slots", "prefixes": prefixes, "drafts": drafts, "tokens": tokens, "context": context, "page": page, "right": right}
    return dict(c, name=name) if name else c


def draw(rng):
    """Sizes between the smallest and the largest listed ones, any head layout and page size."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["attend", "attend", "attend", "append", "append", "pages", "slots"])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    if op == "pages":
        prefixes, drafts, context = log_int(1, 1000), rng.choice([1, 1, 2, 4, 8]), log_int(40, 16384)
        while prefixes > 1 and prefixes * drafts * (context // page + 4) > 2_000_000:
            prefixes = (prefixes + 1) // 2
        return _pages(None, prefixes, drafts, context, page, room=rng.choice([1, 5, 17, 33]), tight=rng.random() < 0.4)
    if op == "slots":
        prefixes, drafts, tokens = log_int(1, 512), rng.choice([1, 1, 4, 8]), log_int(1, 4001)
        prefixes = min(prefixes, max(1, 256_000 // (drafts * tokens)))
        return _slots(None, prefixes, drafts, tokens, tokens + log_int(1, 8000), page, right=rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    dim = rng.choice([32, 64, 64, 96, 128, 128, 128, 192, 256])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16])
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


# ------------------------------------------------------------------------------------------------------ 4-bit values


def _power_of_two(e):
    """2^e in float64 from its bits: exact."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantised(y):
    """(codes [..., D] uint8, scale bytes [..., D / 32] uint8) of float64 or float32 values: the scale is the least 2^e that has the block's
    largest at 7 2^e at most, e in [-120, 125]; an entry becomes the nearest of the 4-bit values, of two as near the one of even code, at most 6."""
    x = y.unflatten(-1, (-1, GROUP))
    most = x.abs().amax(dim=-1)
    m, exponent = torch.frexp(most)                              # most = m 2^exponent, m in [1/2, 1)
    e = torch.where(most > 0, exponent - torch.where(m <= 0.875, 3, 2), -120).clamp(-120, 125)
    t = x.abs() * _power_of_two(-e).to(y.dtype)[..., None]
    code = torch.zeros(t.shape, dtype=torch.uint8, device=y.device)
    for above, or_at in ((0.25, 0.75), (1.25, 1.75), (2.5, 3.5)):
        code += (t > above).to(torch.uint8) + (t >= or_at).to(torch.uint8)
    code += (t > 5.0).to(torch.uint8)
    code |= torch.signbit(x).to(torch.uint8) << 3
    return code.flatten(-2), (e + 127).to(torch.uint8)


def _packed(code):
    """Two codes a byte, the first in the low bits."""
    return code[..., 0::2] | code[..., 1::2] << 4


def _values(packed, scale):
    """float32 values [..., D] of bytes [..., D / 2] and scales [..., D / 32]."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=packed.device)
    x = table[torch.stack((packed & 15, packed >> 4), dim=-1).flatten(-2).int()]
    return (x.unflatten(-1, (-1, GROUP)) * (scale.int() << 23).view(torch.float32)[..., None]).flatten(-2)


# ------------------------------------------------------------------------------------------------------------- inputs


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed) * 1000003 + 31)
    return gen


def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32 if dtype is torch.float32 else dtype) * scale


def _cache(gen, case, pages):
    """k, v [pages, kv_heads, page, dim / 2] and k_scale, v_scale [pages, kv_heads, dim / 32, page], uint8; a page holds its heads one after the
    other, or its tokens."""
    H, P, D = case["kv_heads"], case["page"], case["dim"]
    data, scales = [], []
    for _ in range(2):
        packed = torch.empty((pages, H, P, D // 2), dtype=torch.uint8, device=DEVICE)
        scale = torch.empty((pages, H, P, D // GROUP), dtype=torch.uint8, device=DEVICE)
        step = max(1, (1 << 26) // (H * P * D))
        for at in range(0, pages, step):                         # (a few hundred megabytes of float32 at a time)
            n = min(step, pages - at)
            code, byte = _quantised(torch.randn((n, H, P, D), generator=gen, device=DEVICE))
            packed[at:at + n], scale[at:at + n] = _packed(code), byte
        if case["token_major"]:
            packed = packed.transpose(1, 2).contiguous().transpose(1, 2)
        data.append(packed)
        scales.append(scale.transpose(2, 3).contiguous())
    return data + scales


def prepare(case, seed):
    return {"attend": _prepare_attend, "append": _prepare_append, "pages": _prepare_pages, "slots": _prepare_slots}[case["op"]](case, seed)


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
    ids, place = torch.unique(table, return_inverse=True)        # no more pages than the table uses, and seven
    order = torch.randperm(ids.numel() + 7, generator=gen, device=DEVICE)
    table = order[place].reshape(table.shape).to(torch.int32).contiguous()
    k, v, k_scale, v_scale = _cache(gen, case, ids.numel() + 7)
    q = _normal(gen, (S, T, case["heads"], case["dim"]), dtype, 2.0)
    return {"case": case, "q": q, "k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale, "table": table, "positions": positions,
            "shared_len": whole * P if K > 1 else None, "max_len": context + 8 + T}


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
    k, v, k_scale, v_scale = _cache(gen, case, S * near + 3)
    qkv = _normal(gen, (S, T, H + 2 * G, D), dtype)              # the projections' output: heads of q, k and v side by side
    R = case["rotate"] // 2
    inv_freq = 10000.0 ** (-torch.arange(R, device=DEVICE, dtype=torch.float64) / max(R, 1)) if R else None
    weight = [(1.0 + 0.2 * torch.randn(D, generator=gen, device=DEVICE)).to(dtype) for _ in range(2)] if case["norm"] else [None, None]
    return {"case": case, "q": qkv[:, :, :H], "new_k": qkv[:, :, H:H + G], "new_v": qkv[:, :, H + G:], "k": k, "v": v, "k_scale": k_scale,
            "v_scale": v_scale, "table": table, "positions": positions, "inv_freq": inv_freq, "q_weight": weight[0], "k_weight": weight[1],
            "eps": 1e-6}


STEPS = 16                                                       # of a decoding loop that `run` goes through, one a pass, and begins again


def _prepare_pages(case, seed):
    """A batch in the middle of its work.  In each step a request's text grows by what was accepted of a draft; some requests end, and their
    places get new ones."""
    gen = _generator(seed)
    B, K, P, room, context = (case[k] for k in ("prefixes", "drafts", "page", "room", "context"))

    def whole_number(lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=gen, device=DEVICE)

    length = whole_number(1, max(2, context * 3 // 4), (B,))
    lengths = []
    at = length
    for _ in range(STEPS):
        ends = torch.rand(B, generator=gen, device=DEVICE) < (0.005 if case["tight"] else 0.05)
        new = whole_number(1, max(2, context * 3 // 4), (B,))
        grown = at + whole_number(1, max(2, min(room, 18) // 2 + 1), (B,))
        at = torch.where(at == 0, new, torch.where(ends | (grown > context), 0, grown))
        lengths.append(at)
    width = (context + room + P - 1) // P + 1
    whole, held = length // P, (length + room + P - 1) // P
    each = held + (K - 1) * (held - whole)                       # pages of a request: shared ones, and every draft's own
    begin = torch.cumsum(each, 0) - each
    index = torch.arange(width, device=DEVICE)
    draft = torch.arange(K, device=DEVICE)[:, None]
    place = torch.where((index < whole[:, None, None]) | (draft == 0), index, held[:, None, None] + (draft - 1) * (held - whole)[:, None, None] +
                        index - whole[:, None, None]) + begin[:, None, None]
    used = int(each.sum())
    pages = B * (width + (K - 1) * ((room + P - 1) // P + 2))    # for every request at its longest; `tight`: another program has most of them
    free = int(used * 0.0005) if case["tight"] else pages - used
    order = torch.randperm(pages, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.where(index < held[:, None, None], order[place.clamp(max=pages - 1)], -1).to(torch.int32).reshape(B * K, width).contiguous()
    head = int(used * 0.7)
    ring = torch.roll(torch.cat((order[used:], order[:used])), head).contiguous()        # free pages begin at `head`, round the end
    return {"case": case, "table": table, "ring": ring, "ends": torch.tensor([head, free], dtype=torch.int32, device=DEVICE),
            "held": torch.stack((whole, held), dim=1).to(torch.int32).contiguous(), "lengths": torch.stack(lengths).to(torch.int32),
            "chosen": whole_number(-1, K, (STEPS, B)).to(torch.int32), "step": 0}


def _prepare_slots(case, seed):
    gen = _generator(seed)
    B, K, T, P, context = (case[k] for k in ("prefixes", "drafts", "tokens", "page", "context"))
    width = (context + P - 1) // P
    count = torch.randint(0, T + 1, (B,), generator=gen, device=DEVICE).to(torch.int32)
    count[0] = T
    start = (torch.rand(B, generator=gen, device=DEVICE) * (context - count + 1)).to(torch.int32)
    pages = B * K * width + 5
    table = torch.randperm(pages, generator=gen, device=DEVICE)[:B * K * width].to(torch.int32).reshape(B * K, width)
    holds = (start + count + P - 1) // P
    table = torch.where(torch.arange(width, device=DEVICE) < holds.repeat_interleave(K)[:, None], table, -1).contiguous()
    return {"case": case, "table": table, "pages": pages, "start": start, "count": count}


# ---------------------------------------------------------------------------------------------------------------- run


def run(s):
    op = s["case"]["op"]
    if own:
        return {"attend": _own_attend, "append": _own_append, "pages": _own_pages, "slots": _own_slots}[op](s)
    return {"attend": _plain_attend, "append": _plain_append, "pages": _plain_pages, "slots": _plain_slots}[op](s)


def _handle(s):
    """The handle of the cache is kept between the steps of a decoding loop."""
    import paper_2604_25925_amd as sg
    if "handle" not in s:
        s["handle"] = sg.PackedCache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], DTYPES[s["case"]["dtype"]])
        s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
        s["workspace"] = None
    return sg, s["handle"]


def _own_attend(s):
    """The workspace and the output are kept as well."""
    sg, cache = _handle(s)
    s["out"], s["workspace"] = sg.specgbv_packed_attend(cache, s["q"], s["positions"], window=s["case"]["window"], shared_len=s["shared_len"],
                                                        max_len=s["max_len"], out=s["out"], workspace=s["workspace"])
    return {"out": s["out"]}


def _own_append(s):
    """The new tokens' keys and values are read back: what later steps will see."""
    sg, cache = _handle(s)
    if "seen" not in s:
        s["seen"] = [torch.empty(s["new_k"].shape, dtype=s["new_k"].dtype, device=DEVICE) for _ in range(2)]
    sg.specgbv_packed_append(cache, s["q"], s["new_k"], s["new_v"], s["positions"], inv_freq=s["inv_freq"],
                             interleaved=s["case"]["interleaved"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"], out=s["out"])
    k, v = sg.specgbv_packed_read(cache, s["positions"], k=s["seen"][0], v=s["seen"][1])
    return {"q": s["out"], "k": k, "v": v}


def _own_pages(s):
    import paper_2604_25925_amd as sg
    if "pool" not in s:
        c = s["case"]
        s["pool"] = sg.PagePool(s["table"], s["ring"], s["ends"], s["held"], drafts=c["drafts"], page_size=c["page"])
        s["workspace"] = None
    at = s["step"] % STEPS
    s["step"] += 1
    shared_len, served, s["workspace"] = sg.specgbv_pages_advance(s["pool"], s["lengths"][at], chosen=s["chosen"][at], room=s["case"]["room"],
                                                                  workspace=s["workspace"])
    return {"table": s["table"], "ring": s["ring"], "ends": s["ends"], "held": s["held"], "shared_len": shared_len, "served": served}


def _own_slots(s):
    import paper_2604_25925_amd as sg
    c = s["case"]
    positions, slots = sg.specgbv_slot_map(s["table"], s["start"], s["count"], c["tokens"], page_size=c["page"], pages=s["pages"],
                                           drafts=c["drafts"], right=c["right"])
    return {"positions": positions, "slots": slots}


def _plain_attend(s):
    c, q, pos = s["case"], s["q"], s["positions"].long()
    S, T, H, D = q.shape
    G, P = c["kv_heads"], c["page"]
    width = s["table"].shape[1]
    pages = s["table"].long()
    k, v = (_values(s[x][pages], s[x + "_scale"][pages].transpose(3, 4)).transpose(1, 2).reshape(S, G, width * P, D).contiguous() for x in ("k", "v"))
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

    def turned(x, weight, dtype):
        y = x.to(dtype)
        if weight is not None:
            y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + s["eps"]) * weight.to(dtype)
        R = c["rotate"] // 2
        if R:
            angle = pos.double()[..., None] * s["inv_freq"]                      # [S, T, R]
            cos, sin = angle.cos().to(dtype)[:, :, None], angle.sin().to(dtype)[:, :, None]
            a, b = (y[..., 0:2 * R:2], y[..., 1:2 * R:2]) if c["interleaved"] else (y[..., :R], y[..., R:2 * R])
            pair = (a * cos - b * sin, b * cos + a * sin)
            first = torch.stack(pair, dim=-1).flatten(-2) if c["interleaved"] else torch.cat(pair, dim=-1)
            y = torch.cat((first, y[..., 2 * R:]), dim=-1)
        return y

    out = {"q": (turned(s["q"], s["q_weight"], torch.float32) * there[:, :, None, None]).to(s["q"].dtype)}
    page, slot = s["table"].long().gather(1, (pos // P).clamp(min=0)), pos % P
    for name, y in (("k", turned(s["new_k"], s["k_weight"], torch.float64)), ("v", s["new_v"].float())):
        code, byte = _quantised(y)
        s[name][page[there], :, slot[there]] = _packed(code[there])
        s[name + "_scale"][page[there], :, :, slot[there]] = byte[there]
        seen = _values(s[name][page, :, slot], s[name + "_scale"][page, :, :, slot])
        out[name] = torch.where(there[:, :, None, None], seen, 0.0).to(s["q"].dtype)
    return out


def _plain_pages(s):
    c = s["case"]
    B, K, P = c["prefixes"], c["drafts"], c["page"]
    table, ring = s["table"].view(B, K, -1), s["ring"]
    W, N = table.shape[2], ring.numel()
    at = s["step"] % STEPS
    s["step"] += 1
    length, chosen = s["lengths"][at].long(), s["chosen"][at].long().clamp(0, K - 1)
    whole0, held0 = s["held"].long().unbind(1)
    head, count = s["ends"].long().unbind(0)
    # what the requests ask for
    whole = length.clamp(min=0) // P
    held = torch.where(length > 0, (length + c["room"] + P - 1) // P, 0)
    fits = held <= W
    index = torch.arange(W, device=DEVICE)
    mine = torch.arange(K, device=DEVICE)[None, :, None] == chosen[:, None, None]        # the chosen draft owns the shared pages too
    has = (index >= torch.where(mine, 0, whole0[:, None, None])) & (index < held0[:, None, None])
    wants = (index >= torch.where(mine, 0, whole[:, None, None])) & (index < held[:, None, None])
    gives, takes = (has & ~wants).sum(dim=(1, 2)), (wants & ~has).sum(dim=(1, 2))
    # those that need more than they give back are served in order, until one does not fit: it and such ones behind it stay as they are
    more = torch.where(fits, takes - gives, 0)
    free = count - more.clamp(max=0).sum()
    late = torch.cumsum((torch.cumsum(more.clamp(min=0), 0) > free).int(), 0) > 0
    served = fits & ~((more > 0) & late)
    # pages that are given back go behind the free ones, then pages are taken from the front: by request, the chosen draft first
    order = torch.argsort((~mine).int(), dim=1, stable=True).expand(B, K, W)
    give, take = ((x & served[:, None, None]).gather(1, order).flatten() for x in (has & ~wants, wants & ~has))
    old = table.gather(1, order).flatten()
    given, taken = torch.cumsum(give, 0), torch.cumsum(take, 0)
    behind = torch.where(give, (head + count + given - 1) % N, N)
    ring.copy_(torch.cat((ring, ring[:1])).scatter(0, behind, old)[:N])
    new = torch.where(take, ring[(head + taken - 1) % N], torch.where(give, -1, old)).view(B, K, W)
    new = torch.empty_like(table).scatter_(1, order, new)
    adopted = (index < whole[:, None, None]) & served[:, None, None]
    first = new.gather(1, chosen[:, None, None].expand(B, 1, W))
    table.copy_(torch.where(adopted, first, torch.where(served[:, None, None] & (index >= held[:, None, None]), -1, new)))
    s["ends"].copy_(torch.stack(((head + taken[-1]) % N, count + given[-1] - taken[-1])))
    s["held"].copy_(torch.where(served[:, None], torch.stack((whole, held), dim=1), s["held"]))
    return {"table": s["table"], "ring": ring, "ends": s["ends"], "held": s["held"], "shared_len": (s["held"][:, 0] * P).to(torch.int32),
            "served": torch.where(fits, served.int(), -1).to(torch.int32)}


def _plain_slots(s):
    c = s["case"]
    T, P, K = c["tokens"], c["page"], c["drafts"]
    start, count = s["start"].repeat_interleave(K)[:, None].long(), s["count"].repeat_interleave(K)[:, None].long().clamp(0, T)
    at = torch.arange(T, device=DEVICE) - (T - count if c["right"] else 0)
    there = (at >= 0) & (at < count)
    positions = torch.where(there, start + at, -1)
    page = s["table"].long().gather(1, (positions // P).clamp(0, s["table"].shape[1] - 1))
    held = there & (page >= 0) & (page < s["pages"])
    return {"positions": positions.to(torch.int32), "slots": torch.where(held, page * P + positions % P, -1)}


# --------------------------------------------------------------------------------------------------------------- work


def work(case):
    if case["op"] == "slots":
        n = case["prefixes"] * case["drafts"] * case["tokens"]
        return {"bytes": n * 12 + case["prefixes"] * 8 + 4 * (n // case["page"] + case["prefixes"] * case["drafts"]), "flops": 4 * n}
    if case["op"] == "pages":
        rows = case["prefixes"] * case["drafts"]
        # per request: its state, lengths and answers; per row: about a page given and one taken in a step, the ring read and written
        return {"bytes": case["prefixes"] * 40 + rows * 2 * 4 * 3, "flops": 40 * case["prefixes"] + 8 * rows}
    e = 2 if case["dtype"] == "bf16" else 4
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    T = case["new"]
    held = D / 2 + D / GROUP                                                     # bytes of a key
    if case["op"] == "append":
        tokens = case["sequences"] * (T if T < 3 else 0.67 * T)                  # the others are padding
        return {"bytes": int(tokens * ((2 * H + 4 * G) * D * e + 4 * G * held)), "flops": int(10 * tokens * (H + 2 * G) * D)}
    S, seen = case["prefixes"] * case["drafts"], case["context"]
    if case["window"]:
        seen = min(seen, case["window"])
    if case["ragged"]:
        seen *= 0.5
    kept = case["prefixes"] * seen + (S * (4 + T + case["page"] / 2) if case["drafts"] > 1 else 0)
    return {"bytes": int(2 * S * T * H * D * e + 2 * kept * G * held), "flops": int(4 * S * T * H * D * seen)}


# -------------------------------------------------------------------------------------------------------- in 64 bits


def exact(case, seed):
    if case["op"] not in ("attend", "append"):
        return None                                              # whole numbers
    s = prepare(case, seed)
    return (_exact_attend if case["op"] == "attend" else _exact_append)(case, s)


def _exact_values(packed, scale):
    """float64 [..., D] by the fields of a code: sign, two bits of exponent, one of mantissa."""
    code = torch.empty(packed.shape[:-1] + (2 * packed.shape[-1],), dtype=torch.int64, device=packed.device)
    code[..., 0::2], code[..., 1::2] = packed % 16, packed // 16
    exponent, half = code // 2 % 4, (code % 2).double()
    size = torch.where(exponent == 0, 0.5 * half, (1.0 + 0.5 * half) * 2.0 ** (exponent - 1).double())
    return torch.where(code >= 8, -size, size) * (2.0 ** (scale.double() - 127.0)).repeat_interleave(GROUP, dim=-1)


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
        k, v = (_exact_values(s[x][pages].transpose(0, 1).reshape(G, -1, D // 2)[:, :n],
                              s[x + "_scale"][pages].transpose(0, 1).transpose(2, 3).reshape(G, -1, D // GROUP)[:, :n]) for x in ("k", "v"))
        for t, p in enumerate(row):
            if p < 0:
                continue
            lo = max(0, p + 1 - case["window"]) if case["window"] else 0
            x = q[i, t].reshape(G, H // G, D) * D ** -0.5
            a = torch.softmax(torch.bmm(x, k[:, lo:p + 1].transpose(1, 2).contiguous()), dim=-1)
            out[i, t] = torch.bmm(a, v[:, lo:p + 1].contiguous()).reshape(H, D)
    return {"out": out}


def _exact_held(y):
    """What a float64 head [n, heads, D] is held as: borders between the 4-bit values looked up, the exponent from a logarithm."""
    x = y.unflatten(-1, (-1, GROUP))
    most = x.abs().amax(dim=-1, keepdim=True)
    e = torch.ceil(torch.log2(most.clamp(min=1e-300) / 7.0))
    e = torch.where(most <= 7.0 * 2.0 ** (e - 1), e - 1, torch.where(most > 7.0 * 2.0 ** e, e + 1, e)).clamp(-120, 125)
    size = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=y.device)
    border = (size[1:] + size[:-1]) / 2
    t = (x.abs() / 2.0 ** e).contiguous()
    below, above = torch.searchsorted(border, t), torch.searchsorted(border, t, right=True)
    code = torch.where(below % 2 == 0, below, above)             # on a border: the even one of the two
    return (size[code] * torch.sign(x) * 2.0 ** e).flatten(-2)


def _exact_append(case, s):
    """The rotation as a product of complex numbers."""
    R, pos = case["rotate"] // 2, s["positions"]
    there = (pos >= 0).nonzero()
    where = pos[there[:, 0], there[:, 1]].long()

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

    out = {}
    for name, y in (("q", turned(s["q"], s["q_weight"])), ("k", _exact_held(turned(s["new_k"], s["k_weight"]))),
                    ("v", _exact_held(s["new_v"][there[:, 0], there[:, 1]].double()))):
        out[name] = torch.zeros(pos.shape + y.shape[1:], dtype=torch.float64, device=DEVICE)
        out[name][there[:, 0], there[:, 1]] = y
    return out
