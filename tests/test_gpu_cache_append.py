"""specgbv_cache_append against the definition in float64 (needs an MI355X: run with -m gpu).

Bounds.  With the half step h of the type and e = 2^-24: a head without norm and rotation is copied; a norm is a sum of D squares and a
root (relative error at most (D / 2 + 8) e), and one or two products; a rotated entry is a cos - b sin with cos and sin off by at most 2^-22
absolutely, so it is off by at most (|a| + |b|) (2^-22 + 4 e); the result is rounded once (h)."""
import numpy as np
import pytest

from decoding_util import HALF_STEP, host, make_cache, torch_dtype

pytestmark = pytest.mark.gpu


def _definition(x, positions, inv_freq, interleaved, weight, eps):
    """(y, absolute sums of the rotated pairs) of heads x [S, T, H, D], float64."""
    y = x.astype(np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps) * weight
    mass = np.abs(y)
    R = 0 if inv_freq is None else len(inv_freq)
    if R:
        angle = positions[..., None].astype(np.float64) * inv_freq
        c, s = np.cos(angle)[:, :, None], np.sin(angle)[:, :, None]
        ia, ib = (np.arange(0, 2 * R, 2), np.arange(1, 2 * R, 2)) if interleaved else (np.arange(R), np.arange(R, 2 * R))
        a, b = y[..., ia].copy(), y[..., ib].copy()
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        mass[..., ia] = mass[..., ib] = np.abs(a) + np.abs(b)
    return y, mass


def _bound(y, mass, D, dtype, norm, turned):
    rel = ((D / 2 + 12) * 2.0 ** -24 if norm else 0.0) + (2.0 ** -22 + 4 * 2.0 ** -24 if turned else 0.0)
    return HALF_STEP[dtype] * (np.abs(y) + mass * rel) + mass * rel + 1e-37


def _run(S, T, H, G, D, page, dtype, width, pairs, interleaved=False, norm=False, token_major=False, odd=0, seed=0, in_place=False, spoil=None):
    """`odd`: entries by which q, k and v are shifted in a wider tensor, so that their heads are not 16-byte aligned."""
    import torch
    import paper_2604_25925_amd as sg
    rng = np.random.default_rng(seed + 1000 * D + T)
    dev, dt = torch.device("cuda"), torch_dtype(dtype)
    kc, vc, table = make_cache(rng, S, width, page, G, D, dtype, token_major)
    room = width * page
    positions = np.full((S, T), -1, np.int32)
    for s in range(S):
        n = T if s == 0 else int(rng.integers(0, T + 1))      # padded behind, in front or in between
        where = np.sort(rng.choice(T, n, replace=False))
        start = int(rng.integers(0, room - n + 1))
        positions[s, where] = start + np.arange(n)
    if spoil:
        spoil(positions, table, rng)
    pos = torch.from_numpy(positions).to(dev)
    qkv = torch.from_numpy(rng.normal(0, 1.5, (S, T, H + 2 * G, D + odd)).astype(np.float32)).to(dev).to(dt)[..., odd:]
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + G], qkv[:, :, H + G:]
    freq = torch.from_numpy(10000.0 ** (-np.arange(pairs) / max(pairs, 1))).to(dev) if pairs else None
    w = [torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).to(dev).to(dt) for _ in range(2)] if norm else [None, None]
    eps = 1e-5
    hq, hk, hv, k0, v0 = host(q), host(k), host(v), host(kc), host(vc)
    cache = sg.PagedCache(kc, vc, table)
    out = sg.specgbv_cache_append(cache, q, k, v, pos, inv_freq=freq, interleaved=interleaved, q_weight=w[0], k_weight=w[1], eps=eps,
                                  out=q if in_place else None)
    torch.cuda.synchronize()
    f = None if freq is None else freq.cpu().numpy()
    turned = pairs > 0
    there = positions >= 0
    y, mass = _definition(hq, positions, f, interleaved, None if w[0] is None else host(w[0]), eps)
    got = host(out)
    assert np.all(got[~there] == 0)
    off = np.abs(got - y)[there] / _bound(y, mass, D, dtype, norm, turned)[there]
    assert off.max(initial=0.0) <= 1.0, "q: %.3g times the bound" % off.max()
    y, mass = _definition(hk, positions, f, interleaved, None if w[1] is None else host(w[1]), eps)
    b = _bound(y, mass, D, dtype, norm, turned)
    gk, gv, tab = host(kc), host(vc), table.cpu().numpy()
    stored = np.zeros((k0.shape[0], k0.shape[2]), bool)
    for s in range(S):
        for t in range(T):
            p = positions[s, t]
            if p < 0 or p >= room or not 0 <= tab[s, p // page] < k0.shape[0]:
                continue
            pg, sl = tab[s, p // page], p % page
            stored[pg, sl] = True
            assert np.all(np.abs(gk[pg, :, sl] - y[s, t]) <= b[s, t]), (s, t)
            assert np.array_equal(gv[pg, :, sl], hv[s, t]), (s, t)
    untouched = ~stored
    assert np.array_equal(gk.transpose(0, 2, 1, 3)[untouched], k0.transpose(0, 2, 1, 3)[untouched])      # and nothing else is written
    assert np.array_equal(gv.transpose(0, 2, 1, 3)[untouched], v0.transpose(0, 2, 1, 3)[untouched])
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,pairs,interleaved", [(64, 32, False), (128, 64, False), (128, 64, True), (80, 40, False), (80, 20, False), (96, 24, True),
                                                 (256, 128, False), (256, 64, True), (8, 4, False), (24, 5, False), (40, 3, True), (72, 0, False)])
def test_heads_and_rotations(dtype, D, pairs, interleaved):
    _run(3, 2, 6, 2, D, 16, dtype, 5, pairs, interleaved, norm=False)
    _run(2, 5, 4, 4, D, 8, dtype, 4, pairs, interleaved, norm=True, token_major=True)


@pytest.mark.parametrize("S,T,H,G", [(1, 1, 1, 1), (1, 1, 8, 2), (5, 1, 14, 2), (3, 9, 7, 7), (2, 333, 8, 1), (1, 1200, 3, 1)])
def test_sizes(S, T, H, G):
    _run(S, T, H, G, 64, 32, "bf16", 40, 32, norm=True)


@pytest.mark.parametrize("dtype,odd", [("bf16", 1), ("bf16", 2), ("bf16", 4), ("f32", 1), ("f32", 2)])
@pytest.mark.parametrize("D", [64, 256])
def test_unaligned_heads(dtype, odd, D):
    _run(2, 3, 4, 2, D, 16, dtype, 3, D // 2, norm=True, odd=odd)


def test_in_place():
    _run(2, 7, 4, 2, 128, 16, "bf16", 3, 64, norm=True, in_place=True)


def test_pages_that_are_not_there_and_positions_behind_the_table():
    def spoil(positions, table, rng):
        table[0, 0], table[1, 1], table[2, 2] = -1, 2 ** 31 - 1, -2 ** 31
        table[0, 3] = table.numel() + 3                      # one behind the last page
        positions[0, :4] = [0, 17, 3 * 16, 4 * 16 + 5]
        positions[1, :4] = [16, 31, 5 * 16, 2 ** 31 - 1]     # the last two lie behind the table's five pages
        positions[2, :3] = [2 * 16, 4 * 16 + 15, -2 ** 31]
    _run(3, 4, 4, 2, 64, 16, "bf16", 5, 0, spoil=spoil)


def test_far_positions_keep_their_angles():
    """Positions near 2^20 with frequencies down to 1: angles of 10^6, held to the same bound as near ones."""
    import torch
    import paper_2604_25925_amd as sg
    dev = torch.device("cuda")
    D, page, width = 64, 64, 1 << 14
    kc = torch.zeros((2, 1, page, D), device=dev)
    table = torch.zeros((1, width), dtype=torch.int32, device=dev)
    positions = np.array([[0, 1, 999983, (1 << 20) - 1]], np.int32)
    freq = np.concatenate([np.ones(1), 10000.0 ** (-np.arange(1, 32) / 32)])
    rng = np.random.default_rng(3)
    x = rng.normal(0, 1, (1, 4, 1, D)).astype(np.float32)
    q = torch.from_numpy(x).to(dev)
    out = sg.specgbv_cache_append(sg.PagedCache(kc, kc.clone(), table), q, q, q, torch.from_numpy(positions).to(dev),
                                  inv_freq=torch.from_numpy(freq).to(dev))
    y, mass = _definition(x, positions, freq, False, None, 0.0)
    assert np.all(np.abs(host(out) - y) <= _bound(y, mass, D, "f32", False, True))


def test_caches_beyond_32_bit_offsets():
    """A cache of 2^31 entries and more: the last pages hold what was appended to them."""
    import torch
    import paper_2604_25925_amd as sg
    dev = torch.device("cuda")
    pages, G, page, D = 1100, 8, 1024, 256                   # 2.3e9 entries each
    k = torch.zeros((pages, G, page, D), dtype=torch.bfloat16, device=dev)
    v = torch.zeros_like(k)
    table = torch.tensor([[pages - 1, 3], [pages - 2, 5]], dtype=torch.int32, device=dev)
    x = torch.randn((2, 1, G, D), device=dev).bfloat16()
    y = torch.randn((2, 1, G, D), device=dev).bfloat16()
    pos = torch.tensor([[page - 1], [page]], dtype=torch.int32, device=dev)
    sg.specgbv_cache_append(sg.PagedCache(k, v, table), x, x, y, pos)
    assert torch.equal(k[pages - 1, :, page - 1], x[0, 0]) and torch.equal(v[pages - 1, :, page - 1], y[0, 0])
    assert torch.equal(k[5, :, 0], x[1, 0]) and torch.equal(v[5, :, 0], y[1, 0])
    assert int((k != 0).sum()) == int((x != 0).sum())


def test_replays_of_a_captured_call_on_another_stream():
    import torch
    import paper_2604_25925_amd as sg
    dev = torch.device("cuda")
    rng = np.random.default_rng(5)
    S, T, H, G, D, page = 4, 1, 8, 2, 64, 16
    kc, vc, table = make_cache(rng, S, 4, page, G, D, "bf16")
    cache = sg.PagedCache(kc, vc, table)
    x = torch.randn((S, T, H + 2 * G, D), device=dev).bfloat16()
    pos = torch.zeros((S, T), dtype=torch.int32, device=dev)
    freq = torch.from_numpy(10000.0 ** (-np.arange(32) / 32)).to(dev)
    out = torch.empty((S, T, H, D), dtype=torch.bfloat16, device=dev)
    call = lambda c, o: sg.specgbv_cache_append(c, x[:, :, :H], x[:, :, H:H + G], x[:, :, H + G:], pos, inv_freq=freq, out=o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(cache, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(cache, out)
    for step in range(5):
        x.normal_()
        pos.fill_(step * 9)
        k2, v2, o2 = kc.clone(), vc.clone(), torch.empty_like(out)
        call(sg.PagedCache(k2, v2, table), o2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o2) and torch.equal(kc, k2) and torch.equal(vc, v2)
