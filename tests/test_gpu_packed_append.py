"""Appending to a cache held in 4 bits and reading tokens back, against float64: every code and power, borders between codes, norms and
rotations, what must not be written, strides, blocks that are no numbers."""
import numpy as np
import pytest

import paper_2604_25925_amd as sg
from decoding_util import HALF_STEP, host, torch_dtype
from packed_util import BORDERS, pack, quantise, unpack, values

pytestmark = pytest.mark.gpu


def _dev(x, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(torch_dtype(dtype))


def _cache(gen, S, width, page, G, D, dtype, token_major=False, extra=2):
    """Every byte 0xA5: what a call does not write is seen."""
    import torch
    pages = S * width + extra
    table = torch.from_numpy(gen.permutation(pages)[:S * width].astype(np.int32).reshape(S, width)).cuda()
    data = [torch.full((pages, page, G, D // 2) if token_major else (pages, G, page, D // 2), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2)]
    data = [x.transpose(1, 2) if token_major else x for x in data]
    scale = [torch.full((pages, G, D // 32, page), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2)]
    return sg.PackedCache(*data, *scale, table, torch_dtype(dtype))


def _turned(x, positions, inv_freq, weight, eps, interleaved):
    """Normalised and rotated heads [S, T, H, D] in float64, and the sums of magnitudes behind each entry."""
    y = host(x)
    mass = np.abs(y)
    if weight is not None:
        f = host(weight) / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
        y, mass = y * f, mass * np.abs(f)
    if inv_freq is not None:
        R = inv_freq.shape[0]
        angle = positions[..., None].astype(np.float64) * inv_freq.cpu().numpy()
        cos, sin = np.cos(angle)[:, :, None], np.sin(angle)[:, :, None]
        a, b = (slice(0, 2 * R, 2), slice(1, 2 * R, 2)) if interleaved else (slice(0, R), slice(R, 2 * R))
        out, m = y.copy(), mass.copy()
        out[..., a], out[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
        m[..., a] = m[..., b] = mass[..., a] + mass[..., b]
        y, mass = out, m
    return y, mass


def _run(gen, S, T, H, G, D, page, width, dtype, positions, norm=False, pairs=None, interleaved=False, token_major=False, x=None, label=""):
    """Appends and checks the whole cache's bytes, the queries and what is read back."""
    import torch
    print("case", label, S, T, H, G, D, page, dtype, norm, pairs, interleaved, token_major, flush=True)
    cache = _cache(gen, S, width, page, G, D, dtype, token_major)
    q, k, v = x if x is not None else [_dev(gen.normal(0, 1, (S, T, n, D)), dtype) for n in (H, G, G)]
    pairs = D // 2 if pairs is None else pairs
    inv_freq = torch.from_numpy(10000.0 ** (-np.arange(pairs) / max(pairs, 1))).cuda() if pairs else None
    weight = [_dev(1 + 0.3 * gen.normal(0, 1, D), dtype) if norm else None for _ in range(2)]
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    out = sg.specgbv_packed_append(cache, q, k, v, pos, inv_freq=inv_freq, interleaved=interleaved, q_weight=weight[0], k_weight=weight[1], eps=1e-5)
    p = np.asarray(positions)
    want_q, mass = _turned(q, p, inv_freq, weight[0], 1e-5, interleaved)
    # queries in float32: the norm's sum of D squares, its root and quotient, two products, the turn's three roundings; then the type's own
    err = mass * (D / 2 + 16) * 2.0 ** -24 + HALF_STEP[dtype] * np.abs(want_q) * 1.01 + 1e-37
    got_q = host(out)
    there = p >= 0
    assert not got_q[~there].any()
    assert (np.abs(got_q - want_q) <= err)[there].all(), label
    table = cache.table.cpu().numpy()
    read = sg.specgbv_packed_read(cache, pos)
    for name, y, back in (("k", _turned(k, p, inv_freq, weight[1], 1e-5, interleaved)[0], read[0]), ("v", host(v), read[1])):
        data, scale = getattr(cache, name).cpu().numpy(), getattr(cache, name + "_scale").cpu().numpy()
        code, byte = quantise(y)
        kept = np.full(data.shape, 0xA5, np.uint8), np.full(scale.shape, 0xA5, np.uint8)
        shown = np.zeros(y.shape)
        unsure = np.zeros(y.shape, bool)
        if name == "k":                                       # a rounding in float64 away from a border, or its block's largest from one of the power's
            grid = y.reshape(y.shape[:-1] + (-1, 32))
            most = np.abs(grid).max(-1)
            t = np.abs(grid) / 2.0 ** (byte.astype(np.float64)[..., None] - 127.0)
            near = (np.abs(t[..., None] - BORDERS).min(-1) < 2.0 ** -40) & (pairs > 0 or norm)
            m = np.where(most > 0, most, 1.0)
            near |= ((np.abs(m / 7.0 / 2.0 ** np.round(np.log2(m / 7.0)) - 1.0) < 2.0 ** -40) & (pairs > 0 or norm))[..., None]
            unsure = near.reshape(y.shape)
        for s in range(S):
            for t in range(T):
                n = p[s, t]
                if n < 0 or n >= width * page or not 0 <= table[s, n // page] < cache.pages:
                    continue
                at = table[s, n // page], slice(None), n % page
                kept[0][at] = pack(code[s, t])
                kept[1][at[0], :, :, at[2]] = byte[s, t]
                shown[s, t] = values(code[s, t], byte[s, t])
        if not unsure.any():
            assert (data == kept[0]).all(), (label, name, np.argwhere(data != kept[0])[:5])
            assert (scale == kept[1]).all(), (label, name)
            assert np.array_equal(host(back), shown, equal_nan=True), (label, name)
        else:
            assert ((host(back) == shown) | unsure).all(), (label, name)
    return cache, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 224, 256])
def test_head_dims_norms_and_rotations(D, dtype):
    gen = np.random.default_rng(D)
    for norm in (False, True):
        for pairs in (0, D // 2, D // 4, 3, D // 2 - 1):
            for interleaved in (False, True):
                _run(gen, 2, 3, 4, 2, D, 16, 5, dtype, [[0, 1, 2], [70, -1, 33]], norm, pairs, interleaved, token_major=pairs == 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token_many_tokens_and_far_positions(dtype):
    gen = np.random.default_rng(1)
    _run(gen, 1, 1, 8, 2, 64, 16, 256, dtype, [[4095]])
    _run(gen, 1, 1, 1, 1, 32, 8, 1, dtype, [[0]])
    _run(gen, 1, 1, 4, 1, 128, 128, 1 << 13, dtype, [[(1 << 20) - 1]], norm=True)
    _run(gen, 3, 700, 4, 2, 64, 16, 50, dtype, [[7 + t for t in range(700)], [t if t < 400 else -1 for t in range(700)], [-1] * 300 + list(range(400))], norm=True)
    _run(gen, 2100, 1, 4, 2, 64, 8, 2, dtype, [[int(n)] for n in gen.integers(-1, 16, 2100)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_has_no_place_is_not_written(dtype):
    import torch
    gen = np.random.default_rng(2)
    S, T, H, G, D, page, width = 4, 3, 2, 2, 64, 8, 3
    x = [_dev(gen.normal(0, 1, (S, T, n, D)), dtype) for n in (H, G, G)]
    make = _cache

    def holes(*a, **kw):
        cache = make(*a, **kw)
        cache.table[1, 1] = -1
        cache.table[2, :] = cache.pages
        cache.table[3, 0] = -2 ** 31
        return cache
    try:
        globals()["_cache"] = holes
        _run(gen, S, T, H, G, D, page, width, dtype, [[23, 24, 2 ** 31 - 1], [7, 8, 16], [0, 9, 20], [-1, -2 ** 31, 5]], x=x)
    finally:
        globals()["_cache"] = make
    torch.cuda.synchronize()


def test_ties_borders_and_the_largest_entry():
    """Values in units of the block's power: every border exactly and next to it, and largest entries around 6 and 7, at many powers."""
    gen = np.random.default_rng(3)
    D, S, T, G = 64, 1, 40, 2
    for dtype in ("bf16", "f32"):
        step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -20
        around = np.concatenate([np.array([b, -b, b * (1 + step), b * (1 - step)]) for b in np.concatenate((BORDERS, [5.5, 6.0, 6.5]))])
        y = np.zeros((S, T, G, D))
        for t in range(T):
            unit = 2.0 ** gen.integers(-30, 30)
            for g in range(G):
                for b in range(D // 32):
                    top = gen.choice([4.0, 5.0, 6.0, 6.5, 7.0, 7.0 * (1 + step), 7.5, 3.5, 3.5 * (1 + step)])
                    inside = gen.permutation(around)[:31]
                    y[0, t, g, b * 32:(b + 1) * 32] = unit * gen.permutation(np.append(np.where(np.abs(inside) < top, inside, 0.25), top))
        v = _dev(y, dtype)
        x = [_dev(gen.normal(0, 1, (S, T, 2, D)), dtype), v, v]
        _run(gen, S, T, 2, G, D, 8, 5, dtype, [list(range(T))], pairs=0, x=x, label="borders")


def test_small_large_zero_and_infinite_blocks():
    gen = np.random.default_rng(4)
    D, G = 64, 2
    for dtype in ("bf16", "f32"):
        for size in (0.0, -0.0, 1e-45, 2.0 ** -130, 2.0 ** -122, 2.0 ** -121, 2.0 ** -118, 1e38, 3.3895314e38, float("inf"), float("-inf"), float("nan")):
            y = gen.normal(0, 1, (1, 2, G, D)) if not np.isfinite(size) else np.where(gen.random((1, 2, G, D)) < 0.5, size, -size)
            y[0, 0, 1, 40] = size
            v = _dev(y, dtype)
            x = [_dev(gen.normal(0, 1, (1, 2, 2, D)), dtype), v, v]
            cache, _ = _run(gen, 1, 2, 2, G, D, 8, 1, dtype, [[3, 4]], pairs=0, x=x, label="size %r" % size)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_addresses_and_queries_in_place(dtype):
    import torch
    gen = np.random.default_rng(5)
    S, T, H, G, D, page, width = 2, 5, 4, 2, 64, 16, 4
    positions = [[3 + t for t in range(T)], [40 + t for t in range(T)]]
    room = _dev(gen.normal(0, 1, (S, T, H + 2 * G, D + 9)), dtype)
    for first in (0, 1):                                      # on a border of 16 bytes, and not
        q, k, v = (room[:, :, n:n + m, first:first + D] for n, m in ((0, H), (H, G), (H + G, G)))
        _run(gen, S, T, H, G, D, page, width, dtype, positions, norm=True, x=(q, k, v), label="strided %d" % first)
        wide = torch.from_numpy(10000.0 ** (-np.arange(D // 2) / (D // 2))).cuda()
        pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
        cache = _cache(gen, S, width, page, G, D, dtype)
        apart = sg.specgbv_packed_append(cache, q, k, v, pos, inv_freq=wide)
        kept = room.clone()
        same = kept[:, :, :H, first:first + D]
        sg.specgbv_packed_append(cache, same, kept[:, :, H:H + G, first:first + D], kept[:, :, H + G:, first:first + D], pos, inv_freq=wide, out=same)
        assert torch.equal(same, apart)
        kept[:, :, :H, first:first + D] = room[:, :, :H, first:first + D]
        assert torch.equal(kept, room)


def test_read_strides_padding_and_holes():
    import torch
    gen = np.random.default_rng(6)
    for dtype in ("bf16", "f32"):
        S, T, H, G, D, page, width = 2, 4, 2, 3, 96, 8, 3
        cache = _cache(gen, S, width, page, G, D, dtype)
        for x in (cache.k, cache.v):
            x.copy_(torch.from_numpy(gen.integers(0, 256, tuple(x.shape), dtype=np.uint8)))
        for x in (cache.k_scale, cache.v_scale):
            x.copy_(torch.from_numpy(gen.integers(100, 140, tuple(x.shape), dtype=np.uint8)))
        cache.table[0, 1] = -1
        cache.table[1, 2] = cache.pages
        p = [[0, 9, -1, 17], [23, 15, 24, 2 ** 31 - 1]]
        pos = torch.tensor(p, dtype=torch.int32, device="cuda")
        room = [torch.full((S, T, G, D + 5), 3.0, dtype=torch_dtype(dtype), device="cuda") for _ in range(2)]
        table = cache.table.cpu().numpy()
        for outs in ((None, None), (room[0][..., 2:D + 2], room[1][..., :D])):
            k, v = sg.specgbv_packed_read(cache, pos, k=outs[0], v=outs[1])
            for got, x, s in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
                want = np.zeros((S, T, G, D))
                whole = values(unpack(x.cpu().numpy()), np.swapaxes(s.cpu().numpy(), 2, 3))
                for i in range(S):
                    for t in range(T):
                        n = p[i][t]
                        if 0 <= n < width * page and 0 <= table[i, n // page] < cache.pages:
                            want[i, t] = whole[table[i, n // page], :, n % page]
                assert (host(got) == want).all()
        assert (room[0][..., :2] == 3).all() and (room[0][..., D + 2:] == 3).all() and (room[1][..., D:] == 3).all()


def test_appended_tokens_in_a_captured_graph():
    import torch
    gen = np.random.default_rng(7)
    S, T, H, G, D, page, width = 3, 1, 4, 2, 64, 16, 4
    cache, other = (_cache(np.random.default_rng(8), S, width, page, G, D, "bf16") for _ in range(2))
    x = [_dev(gen.normal(0, 1, (S, T, n, D)), "bf16") for n in (H, G, G)]
    pos = torch.tensor([[5], [17], [40]], dtype=torch.int32, device="cuda")
    inv = torch.from_numpy(10000.0 ** (-np.arange(D // 2) / (D // 2))).cuda()
    out = torch.empty_like(x[0])
    sg.specgbv_packed_append(cache, *x, pos, inv_freq=inv, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sg.specgbv_packed_append(cache, *x, pos, inv_freq=inv, out=out)
        back = sg.specgbv_packed_read(cache, pos)
    for turn in range(4):
        x[1].copy_(_dev(gen.normal(0, 1, (S, T, G, D)), "bf16"))
        pos += 1
        graph.replay()
        torch.cuda.synchronize()
        want = sg.specgbv_packed_append(other, *x, pos, inv_freq=inv)
        assert torch.equal(want, out)
        for a, b in zip(back, sg.specgbv_packed_read(other, pos)):
            assert torch.equal(a, b), turn
