"""Attention over a cache held in 4 bits against float64: head layouts, pages, windows, drafts of a prefix, lengths of none and one, what
is masked, pages that are not there, blocks that are no numbers, strides, far pages, streams and graphs."""
import numpy as np
import pytest

import paper_2604_25925_amd as sg
from decoding_util import host, torch_dtype
from packed_util import check, dense, make_packed

pytestmark = pytest.mark.gpu


def _q(gen, shape, dtype, scale=1.0):
    import torch
    return torch.from_numpy((gen.normal(0, scale, shape)).astype(np.float32)).cuda().to(torch_dtype(dtype))


def _positions(rows):
    import torch
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


def _label(*a):
    print("case", *a, flush=True)
    return " ".join(map(str, a))


@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_dims(D, dtype):
    gen = np.random.default_rng(D)
    for S, T, H, G, page, width, token_major in ((3, 1, 8, 2, 16, 6, False), (2, 5, 14, 2, 8, 9, True), (1, 9, 3, 3, 64, 3, False), (2, 2, 20, 1, 24, 5, True)):
        label = _label(D, dtype, S, T, H, G, page, token_major)
        cache = make_packed(gen, S, width, page, G, D, dtype, token_major)
        q = _q(gen, (S, T, H, D), dtype)
        last = gen.integers(T, width * page, S)
        positions = _positions([[int(n) - T + 1 + t for t in range(T)] for n in last])
        out, _ = sg.specgbv_packed_attend(cache, q, positions)
        check(out, cache, q, positions, dtype, label=label)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 513, 1000, 2047])
def test_lengths(length, dtype):
    gen = np.random.default_rng(length)
    for D, H, G, S in ((128, 8, 2, 1), (64, 6, 1, 2)):
        label = _label(length, dtype, D)
        cache = make_packed(gen, S, (length + 15) // 16, 16, G, D, dtype)
        q = _q(gen, (S, 1, H, D), dtype)
        positions = _positions([[length - 1]] * S)
        out, _ = sg.specgbv_packed_attend(cache, q, positions)
        check(out, cache, q, positions, dtype, label=label)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 1000])
def test_windows(window, dtype):
    gen = np.random.default_rng(window)
    S, T, H, G, D, page, width = 4, 5, 6, 2, 64, 16, 40
    cache = make_packed(gen, S, width, page, G, D, dtype)
    q = _q(gen, (S, T, H, D), dtype)
    positions = _positions([[n + t for t in range(T)] for n in (0, 17, 300, 630)])
    out, _ = sg.specgbv_packed_attend(cache, q, positions, window=window)
    check(out, cache, q, positions, dtype, window=window, label=_label(window, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_and_prompts(dtype):
    """Rows of their own for every wave, several row blocks, with and without parts."""
    gen = np.random.default_rng(5)
    for S, T, H, G, D, length in ((1, 70, 8, 1, 64, 90), (2, 33, 16, 2, 128, 300), (1, 130, 4, 1, 256, 140), (1, 300, 2, 2, 64, 300), (3, 17, 64, 4, 96, 700)):
        label = _label(dtype, S, T, H, G, D, length)
        width = (length + 31) // 32
        cache = make_packed(gen, S, width, 32, G, D, dtype)
        q = _q(gen, (S, T, H, D), dtype)
        positions = _positions([[length - T + t for t in range(T)]] * S)
        out, _ = sg.specgbv_packed_attend(cache, q, positions)
        check(out, cache, q, positions, dtype, label=label)


@pytest.mark.parametrize("S", [64, 65, 130, 300])
def test_many_sequences(S):
    gen = np.random.default_rng(S)
    for longest in (40, 330):
        label = _label(S, longest)
        cache = make_packed(gen, S, (longest + 7) // 8, 8, 2, 64)
        q = _q(gen, (S, 1, 4, 64), "bf16")
        positions = _positions([[int(n)] for n in gen.integers(-1, longest, S)])
        out, _ = sg.specgbv_packed_attend(cache, q, positions)
        check(out, cache, q, positions, "bf16", label=label)


def _share(cache, drafts, whole):
    """The first `whole[b]` pages of a prefix's drafts are its first draft's."""
    table = cache.table
    for b, n in enumerate(whole):
        table[b * drafts:(b + 1) * drafts, :n] = table[b * drafts, :n]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,K,T,H,G,D,page", [(3, 4, 1, 8, 2, 64, 16), (2, 8, 3, 8, 2, 128, 8), (5, 2, 9, 4, 4, 64, 32), (1, 8, 9, 16, 2, 128, 16), (70, 2, 1, 4, 1, 64, 8),
                                              (2, 3, 2, 4, 1, 256, 16)])
@pytest.mark.parametrize("window", [0, 50])
def test_drafts_of_a_prefix(B, K, T, H, G, D, page, dtype, window):
    import torch
    gen = np.random.default_rng(B * 100 + K)
    width = 300 // page + 2
    cache = make_packed(gen, B * K, width, page, G, D, dtype)
    whole = gen.integers(0, 280 // page, B)
    whole[0] = 0
    _share(cache, K, whole)
    positions = _positions([[int(whole[b]) * page + int(gen.integers(0, page)) + t if gen.random() > 0.1 else -1 for t in range(T)] for b in range(B) for _ in range(K)])
    q = _q(gen, (B * K, T, H, D), dtype)
    shared = torch.from_numpy((whole * page).astype(np.int32)).cuda()
    label = _label(B, K, T, H, G, D, page, dtype, window)
    out, ws = sg.specgbv_packed_attend(cache, q, positions, window=window, shared_len=shared)
    check(out, cache, q, positions, dtype, window=window, label=label)
    for max_len in (40, 300):                                # the hint changes the split and nothing else; the workspace serves all
        again, _ = sg.specgbv_packed_attend(cache, q, positions, window=window, shared_len=shared, max_len=max_len, workspace=ws)
        check(again, cache, q, positions, dtype, window=window, label=label + " max_len %d" % max_len)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,K,T,H,G,D,page", [(3, 4, 1, 8, 2, 64, 16), (2, 8, 3, 8, 2, 128, 8), (2, 2, 9, 4, 4, 64, 32), (1, 8, 9, 16, 2, 128, 16), (70, 2, 1, 4, 1, 64, 8),
                                              (2, 3, 2, 4, 1, 256, 16)])
@pytest.mark.parametrize("window", [0, 50])
def test_drafts_of_a_prefix_in_a_table_for_long_ones(B, K, T, H, G, D, page, dtype, window):
    """Tables of more than 2560 tokens: the drafts' shared pages are read once, also where a prefix is short, empty or all that a draft has."""
    import torch
    gen = np.random.default_rng(B * 100 + K + 7)
    width = 2700 // page + 1
    cache = make_packed(gen, B * K, width, page, G, D, dtype)
    whole = gen.integers(0, (2680 if B < 5 else 400) // page, B)
    whole[0] = 0
    whole[-1] = 100 // page
    if B > 2:
        whole[1] = width - 1
    _share(cache, K, whole)
    shared = whole * page
    rows = [[int(shared[b]) + int(gen.integers(0, page)) + t if gen.random() > 0.1 else -1 for t in range(T)] for b in range(B) for _ in range(K)]
    rows[0] = [-1] * T                                       # a draft of padding alone
    rows[-1] = [int(shared[-1]) - 1] * T                     # one that has nothing but the prefix
    positions = _positions(rows)
    q = _q(gen, (B * K, T, H, D), dtype)
    out, _ = sg.specgbv_packed_attend(cache, q, positions, window=window, shared_len=torch.from_numpy(shared.astype(np.int32)).cuda())
    check(out, cache, q, positions, dtype, window=window, label=_label(B, K, T, H, G, D, page, dtype, window))


@pytest.mark.parametrize("S,T,H,G,D,length,dtype", [(70, 1, 4, 1, 64, 3000, "bf16"), (66, 1, 4, 1, 64, 3000, "f32"), (1, 70, 2, 1, 128, 2900, "bf16"), (2, 100, 4, 2, 64, 1500, "f32")])
def test_more_units_than_are_weighed_in_parts(S, T, H, G, D, length, dtype):
    """Parts of equal lengths: more than 64 sequences, or prompts in chunks, over long tables, some of which hold little."""
    gen = np.random.default_rng(S + T)
    cache = make_packed(gen, S, (length + 15) // 16, 16, G, D, dtype)
    q = _q(gen, (S, T, H, D), dtype)
    last = [length - 1] + [int(n) for n in gen.integers(T - 1, length, S - 1)]
    positions = _positions([[n - T + 1 + t for t in range(T)] for n in last])
    for window in (0, 1200):
        out, _ = sg.specgbv_packed_attend(cache, q, positions, window=window)
        check(out, cache, q, positions, dtype, window=window, label=_label(S, T, H, G, D, length, dtype, window))


@pytest.mark.parametrize("S,T,H,G,D,length,dtype", [(600, 1, 4, 2, 64, 100, "bf16"), (530, 1, 4, 2, 64, 100, "f32"), (300, 1, 8, 4, 128, 260, "bf16"), (140, 9, 8, 4, 128, 130, "f32"),
                                                    (300, 1, 4, 2, 256, 150, "bf16"), (260, 1, 2, 2, 256, 70, "f32"), (200, 9, 16, 4, 128, 50, "bf16")])
@pytest.mark.parametrize("window", [0, 33])
def test_more_sequences_than_workgroups_at_once(S, T, H, G, D, length, dtype, window):
    """Each wave by itself, in workgroups whose last waves have nothing."""
    gen = np.random.default_rng(S + D)
    page = 16 if D == 64 else 8
    cache = make_packed(gen, S, (length + page - 1) // page, page, G, D, dtype)
    q = _q(gen, (S, T, H, D), dtype)
    positions = _positions([[int(n) - T + 1 + t if n >= 0 else -1 for t in range(T)] for n in gen.integers(-1, length, S)])
    out, _ = sg.specgbv_packed_attend(cache, q, positions, window=window)
    check(out, cache, q, positions, dtype, window=window, label=_label(S, T, H, G, D, length, dtype, window))


@pytest.mark.parametrize("B,K,T,H,G,D,width,dtype", [(3, 4, 3, 8, 2, 64, 20, "bf16"), (2, 3, 9, 8, 2, 128, 170, "bf16"), (2, 4, 2, 4, 1, 64, 170, "f32"), (24, 8, 1, 8, 8, 64, 45, "bf16")])
def test_shared_lengths_that_are_no_whole_pages(B, K, T, H, G, D, width, dtype):
    """Drafts whose tables are the same: whatever number of tokens is said to be shared, also below 0 and behind what queries see or the table holds, the result is that of their tokens."""
    import torch
    gen = np.random.default_rng(B + D)
    page = 16
    cache = make_packed(gen, B * K, width, page, G, D, dtype)
    _share(cache, K, [width] * B)
    positions = _positions([[int(n) + t for t in range(T)] for n in gen.integers(0, width * page - T, B * K)])
    q = _q(gen, (B * K, T, H, D), dtype)
    for said in ([-5, 7, 10 ** 9], [0, width * page, 33], [2 ** 31 - 1, -2 ** 31, width * page - 1]):
        shared = torch.tensor((said * B)[:B], dtype=torch.int32, device="cuda")
        out, _ = sg.specgbv_packed_attend(cache, q, positions, shared_len=shared)
        check(out, cache, q, positions, dtype, label=_label(B, K, T, D, dtype, said))


def test_long_sequences_in_parts():
    gen = np.random.default_rng(8)
    for S, T, H, G, D, length, hint in ((1, 1, 8, 2, 128, 20000, None), (2, 3, 4, 1, 64, 9000, 100), (1, 40, 8, 1, 128, 5000, None)):
        label = _label(S, T, H, G, D, length)
        cache = make_packed(gen, S, (length + 63) // 64, 64, G, D)
        q = _q(gen, (S, T, H, D), "bf16")
        positions = _positions([[length - 1 - s * 1234 - T + 1 + t for t in range(T)] for s in range(S)])
        out, _ = sg.specgbv_packed_attend(cache, q, positions, max_len=hint)
        check(out, cache, q, positions, "bf16", label=label)


def test_padding_empty_sequences_and_positions_behind_the_table():
    gen = np.random.default_rng(3)
    S, T, H, G, D, page, width = 6, 4, 4, 2, 64, 8, 4
    for dtype in ("bf16", "f32"):
        cache = make_packed(gen, S, width, page, G, D, dtype)
        q = _q(gen, (S, T, H, D), dtype)
        positions = _positions([[-1, -1, -1, -1], [0, 1, 2, 3], [-1, 5, -1, 6], [31, 32, 1000, 2 ** 31 - 1], [-2 ** 31, 0, -7, 30], [-1, -1, -1, 0]])
        out, _ = sg.specgbv_packed_attend(cache, q, positions)
        check(out, cache, q, positions, dtype, label=_label(dtype))
        assert not host(out)[0].any()


def test_pages_that_are_not_there():
    import torch
    gen = np.random.default_rng(4)
    S, T, H, G, D, page, width = 3, 2, 4, 2, 64, 8, 9
    for bad in (-1, -2 ** 31, 2 ** 31 - 1, None):
        cache = make_packed(gen, S, width, page, G, D)
        bad = cache.pages if bad is None else bad
        cache.table[0, 2] = bad
        cache.table[1, :] = bad
        cache.table[2, 8] = bad
        q = _q(gen, (S, T, H, D), "bf16")
        positions = _positions([[60, 61], [5, 70], [66, 67]])
        out, _ = sg.specgbv_packed_attend(cache, q, positions)
        check(out, cache, q, positions, "bf16", label=_label(bad))
        assert not host(out)[1].any()
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,T,H", [(64, 3, 4), (128, 3, 4), (256, 2, 2), (96, 40, 8)])
def test_blocks_that_are_no_numbers_stay_where_they_are_seen(D, T, H, dtype):
    """Powers of 255 in unused pages and slots, behind every query and in front of the window are of no matter; a value's block that some queries
    see makes its 32 entries of those NaN and no others; a key's block makes all of them NaN."""
    gen = np.random.default_rng(D + T)
    S, G, page, width, window = 2, 2, 16, 8, 60
    cache = make_packed(gen, S, width, page, G, D, dtype)
    q = _q(gen, (S, T, H, D), dtype)
    positions = _positions([[n + t for t in range(T)] for n in (70, 64)])
    table = cache.table.cpu().numpy()
    unused = np.setdiff1d(np.arange(cache.pages), table)
    for scale in (cache.k_scale, cache.v_scale):
        for p in unused:
            scale[int(p)] = 255
        for s, n in enumerate((70, 64)):
            for at in range(width * page):
                if at > n + T - 1 or at <= n - window:       # seen by no query
                    scale[int(table[s, at // page]), :, :, at % page] = 255
    label = _label(D, T, H, dtype)
    clean, _ = sg.specgbv_packed_attend(cache, q, positions, window=window)
    assert np.isfinite(host(clean)).all(), label
    kept = {x: getattr(cache, x + "_scale").clone() for x in ("k", "v")}
    for s in (cache.k_scale, cache.v_scale):
        s[s == 255] = 127
    check(clean, cache, q, positions, dtype, window=window, label=label)
    cache.v_scale.copy_(kept["v"])
    cache.k_scale.copy_(kept["k"])
    t0 = T // 2
    at, block, g = 70 + t0, D // 32 - 1, 1                   # queries t >= t0 of sequence 0 see this token
    cache.v_scale[int(table[0, at // page]), g, block, at % page] = 255
    got = host(sg.specgbv_packed_attend(cache, q, positions, window=window)[0])
    nan = np.zeros(got.shape, bool)
    nan[0, t0:, g * (H // G):(g + 1) * (H // G), block * 32:] = True
    assert (np.isnan(got) == nan).all(), label
    assert (got[~nan] == host(clean)[~nan]).all(), label
    cache.v_scale.copy_(kept["v"])
    cache.k_scale[int(table[0, at // page]), g, 0, at % page] = 255
    got = host(sg.specgbv_packed_attend(cache, q, positions, window=window)[0])
    nan[:] = False
    nan[0, t0:, g * (H // G):(g + 1) * (H // G)] = True
    assert (np.isnan(got) == nan).all(), label
    assert (got[~nan] == host(clean)[~nan]).all(), label


def test_queries_of_large_and_small_scores():
    """Scores far apart, all far below zero and near the type's range: the running reference moves and nothing overflows."""
    gen = np.random.default_rng(9)
    S, T, H, G, D, page, width = 2, 2, 4, 1, 64, 16, 20
    for dtype in ("bf16", "f32"):
        for size in (1e-30, 1e-3, 30.0, 3e3, 1e6):
            cache = make_packed(gen, S, width, page, G, D, dtype)
            q = _q(gen, (S, T, H, D), dtype, size)
            positions = _positions([[300, 301], [100, 101]])
            scale = 0.125
            out, _ = sg.specgbv_packed_attend(cache, q, positions, scale=scale)
            k, v = dense(cache)
            if size <= 30.0:
                check(out, cache, q, positions, dtype, scale=scale, label=_label(dtype, size))
            else:                                            # one key has all the weight, or few that lie close: a mean of values
                assert np.isfinite(host(out)).all() and np.abs(host(out)).max() <= np.abs(v).max() * (1 + 2.0 ** -8)


def test_infinite_queries_of_float32_are_not_made_nan_by_their_operands():
    """-inf times keys of one sign gives scores of -inf for all keys but those that are 0 there."""
    import torch
    gen = np.random.default_rng(10)
    cache = make_packed(gen, 1, 2, 16, 1, 64, "f32")
    cache.k[:] = 0x22                                        # every entry 1
    cache.k_scale[:] = 127
    q = torch.zeros((1, 1, 1, 64), device="cuda")
    q[..., 3] = float("inf")
    positions = _positions([[20]])
    assert np.isnan(host(sg.specgbv_packed_attend(cache, q, positions)[0])).all()         # the sum of infinite weights
    q[..., 3] = float("-inf")
    got = host(sg.specgbv_packed_attend(cache, q, positions)[0])
    assert (got == 0).all()                                  # every weight is 0
    q[..., 3] = 3.4028234e38                                 # rounding this to bfloat16 would make it infinite
    q[..., 4] = -3.4028234e38
    got = host(sg.specgbv_packed_attend(cache, q, positions)[0])
    ref = dense(cache)[1][cache.table.cpu().numpy()[0]][:, 0].reshape(-1, 64)[:21].mean(0)
    assert np.abs(got[0, 0, 0] - ref).max() <= 64 * 2.0 ** -23 * 6


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_addresses(dtype):
    import torch
    gen = np.random.default_rng(11)
    S, T, H, G, D, page, width = 2, 3, 4, 2, 64, 16, 6
    cache = make_packed(gen, S, width, page, G, D, dtype)
    room = _q(gen, (S, T, H + 3, D + 9), dtype)
    rows = torch.full((S, T + 4), 7, dtype=torch.int32, device="cuda")
    rows[:, :T] = _positions([[50, 51, 52], [90, 91, 92]])
    positions = rows[:, :T]
    for q in (room[:, :, 1:H + 1, 1:D + 1], room.transpose(0, 1).contiguous().transpose(0, 1)[:, :, :H, :D]):
        back = torch.full((S, T, H + 1, D + 5), 3.0, dtype=torch_dtype(dtype), device="cuda")
        out = back[:, :, :H, 3:D + 3]
        sg.specgbv_packed_attend(cache, q, positions, out=out)
        check(out, cache, q, positions, dtype, label=_label(dtype, q.stride()))
        assert (back[:, :, H] == 3).all() and (back[..., :3] == 3).all() and (back[..., D + 3:] == 3).all()


@pytest.mark.parametrize("way,page", [(way, page) for way in ("one pass", "parts", "waves") for page in (32, 16, 8)] + [("one pass", "far"), ("parts", "far")])
@pytest.mark.parametrize("dtype,D,T", [("bf16", 64, 5), ("bf16", 64, 17), ("bf16", 64, 40), ("bf16", 128, 5), ("bf16", 128, 17), ("bf16", 128, 40), ("bf16", 256, 5),
                                       ("bf16", 256, 17), ("f32", 64, 5), ("f32", 64, 17), ("f32", 128, 5), ("f32", 128, 17), ("f32", 256, 5)])
def test_rows_pages_and_ways(dtype, D, T, way, page):
    """16, 32 and 64 rows at once; pages of whole, half and quarter tiles; one pass, parts, and (with more rows than workgroups) waves by themselves."""
    gen = np.random.default_rng(D + T)
    far = page == "far"
    page = 8 if far else page
    S, G, length = {"one pass": (3, 2, 90), "parts": (2, 1, 2500), "waves": (265, 4, 60)}[way]
    width = (length + page - 1) // page
    stride = None
    if far:
        stride = 2 ** 32 // (S * width - 2) // 16 * 16
    cache = make_packed(gen, S, width, page, G, D, dtype, extra=1, page_stride=stride)
    q = _q(gen, (S, T, G, D), dtype)
    positions = _positions([[int(n) - T + 1 + t for t in range(T)] for n in gen.integers(length // 2, length, S)])
    out, _ = sg.specgbv_packed_attend(cache, q, positions)
    check(out, cache, q, positions, dtype, label=_label(dtype, D, T, way, page, far))


@pytest.mark.parametrize("page", [32, 16, 8, "far"])
@pytest.mark.parametrize("dtype,D,T", [("bf16", 64, 5), ("bf16", 64, 17), ("bf16", 128, 5), ("bf16", 128, 17), ("bf16", 256, 5), ("f32", 64, 5), ("f32", 64, 17), ("f32", 128, 5),
                                       ("f32", 256, 5)])
def test_workgroups_that_fill_a_compute_unit(dtype, D, T, page):
    """About as many rows of workgroups as compute units, over lengths that parts would be made of; sequences with little or nothing among them."""
    gen = np.random.default_rng(D + T + 1)
    far = page == "far"
    page = 8 if far else page
    S, G, length = 40, 2, 1060
    width = (length + page - 1) // page
    cache = make_packed(gen, S, width, page, G, D, dtype, extra=1, page_stride=2 ** 32 // (S * width - 2) // 16 * 16 if far else None)
    q = _q(gen, (S, T, G, D), dtype)
    last = [length - 1, T - 1, -1, 40] + [int(n) for n in gen.integers(T - 1, length, S - 4)]
    positions = _positions([[max(n - T + 1 + t, -1) for t in range(T)] for n in last])
    label = _label(dtype, D, T, page, far)
    out, ws = sg.specgbv_packed_attend(cache, q, positions)
    check(out, cache, q, positions, dtype, label=label)
    for window, max_len in ((700, None), (0, 300)):          # (the workspace serves the parts of other lengths too)
        out, _ = sg.specgbv_packed_attend(cache, q, positions, window=window, max_len=max_len, workspace=ws)
        check(out, cache, q, positions, dtype, window=window, label=label + " %d %s" % (window, max_len))


@pytest.mark.parametrize("B,K,T,H,G,D,page,dtype", [(24, 8, 1, 8, 8, 64, 16, "bf16"), (16, 8, 1, 16, 8, 128, 16, "f32"), (16, 8, 3, 8, 8, 128, 32, "bf16"), (16, 8, 2, 8, 8, 256, 8, "bf16"),
                                                    (12, 16, 1, 16, 8, 64, 8, "f32"), (16, 8, 4, 8, 8, 64, 64, "bf16")])
def test_drafts_in_workgroups_that_fill_a_compute_unit(B, K, T, H, G, D, page, dtype):
    import torch
    gen = np.random.default_rng(B + K + D)
    width = 900 // page + 2
    cache = make_packed(gen, B * K, width, page, G, D, dtype)
    whole = gen.integers(0, 900 // page, B)
    whole[0], whole[1] = 0, width - 1
    _share(cache, K, whole)
    shared = whole * page
    rows = [[int(shared[b]) + int(gen.integers(0, page)) + t if gen.random() > 0.1 else -1 for t in range(T)] for b in range(B) for _ in range(K)]
    rows[0] = [-1] * T
    rows[-1] = [max(int(shared[-1]) - 1, 0)] * T
    positions = _positions(rows)
    q = _q(gen, (B * K, T, H, D), dtype)
    shared = torch.from_numpy(shared.astype(np.int32)).cuda()
    label = _label(B, K, T, H, G, D, page, dtype)
    ws = None
    for window, max_len in ((0, None), (60, None), (0, 2000), (0, 200)):
        out, used = sg.specgbv_packed_attend(cache, q, positions, window=window, shared_len=shared, max_len=max_len, workspace=ws)
        ws = used if ws is None else ws
        check(out, cache, q, positions, dtype, window=window, label=label + " %d %s" % (window, max_len))


@pytest.mark.parametrize("tiles,way,page", [(tiles, way, page) for tiles, way in ((2, "one pass"), (2, "parts"), (2, "filled"), (2, "waves"), (4, "one pass"), (4, "parts"))
                                            for page in (32, 16, 8, "far") if (way, page) != ("waves", "far")])         # (far pages of 8 tokens are not taken by waves alone)
@pytest.mark.parametrize("D", [64, 128])
def test_many_rows_of_bfloat16_at_once(D, tiles, way, page):
    """So many rows that a wave takes 32 or 64 of them, in each way in which it does."""
    gen = np.random.default_rng(D + tiles)
    far = page == "far"
    page = 8 if far else page
    S, T, length = {(2, "one pass"): (129, 1, 90), (2, "parts"): (129, 1, 1900), (2, "filled"): (129, 1, 1060), (2, "waves"): (1024, 1, 60), (4, "one pass"): (128, 4, 320),
                    (4, "parts"): (128, 4, 1100)}[tiles, way]
    width = (length + page - 1) // page
    cache = make_packed(gen, S, width, page, 1, D, extra=1, page_stride=2 ** 32 // (S * width - 2) // 16 * 16 + 16 if far else None)
    q = _q(gen, (S, T, 32, D), "bf16")
    last = [length - 1, T - 1, -1, 40] + [int(n) for n in gen.integers(T - 1, length, S - 4)]
    positions = _positions([[max(n - T + 1 + t, -1) for t in range(T)] for n in last])
    for window in (0, length - 7):
        out, _ = sg.specgbv_packed_attend(cache, q, positions, window=window)
        check(out, cache, q, positions, "bf16", window=window, label=_label(D, tiles, way, page, far, window))


@pytest.mark.parametrize("D,page,S", [(64, 32, 2), (128, 8, 2), (256, 32, 2), (64, 24, 2)])
def test_pages_of_other_sizes_more_than_2_to_the_32_bytes_apart(D, page, S):
    gen = np.random.default_rng(D + page)
    T, H, G, width = 2, 4, 2, 1
    cache = make_packed(gen, S, width, page, G, D, extra=1, page_stride=2 ** 31 - 16)
    cache.table[0, 0], cache.table[1, 0] = 2, 0
    q = _q(gen, (S, T, H, D), "bf16")
    positions = _positions([[5, 6], [page - 2, page - 1]])
    out, _ = sg.specgbv_packed_attend(cache, q, positions)
    check(out, cache, q, positions, "bf16", label=_label(D, page))


@pytest.mark.parametrize("D", [64, 128])
def test_pages_more_than_2_to_the_32_bytes_apart(D):
    gen = np.random.default_rng(12)
    S, T, H, G, page, width = 2, 2, 4, 2, 16, 1
    cache = make_packed(gen, S, width, page, G, D, extra=1, page_stride=2 ** 31 - 16)
    cache.table[0, 0], cache.table[1, 0] = 2, 0
    q = _q(gen, (S, T, H, D), "bf16")
    positions = _positions([[9, 10], [14, 15]])
    out, _ = sg.specgbv_packed_attend(cache, q, positions)
    check(out, cache, q, positions, "bf16", label=_label(D))


def test_another_stream_and_graphs_that_share_a_workspace():
    import torch
    gen = np.random.default_rng(13)
    S, T, H, G, D, page, width = 2, 1, 8, 2, 128, 16, 130
    cache = make_packed(gen, S, width, page, G, D)
    q = [_q(gen, (S, T, H, D), "bf16") for _ in range(2)]
    positions = _positions([[2000], [1500]])
    want = [sg.specgbv_packed_attend(cache, x, positions)[0] for x in q]
    _, ws = sg.specgbv_packed_attend(cache, q[0], positions)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = sg.specgbv_packed_attend(cache, q[1], positions)
    side.synchronize()
    assert torch.equal(got, want[1])
    torch.cuda.synchronize()
    graphs, outs = [], [torch.empty_like(x) for x in q]
    for x, o in zip(q, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sg.specgbv_packed_attend(cache, x, positions, out=o, workspace=ws)
        graphs.append(graph)
    for turn in range(4):
        for o in outs:
            o.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        eager, _ = sg.specgbv_packed_attend(cache, q[0], positions)
        assert torch.equal(eager, want[0])
        for o, w in zip(outs, want):
            assert torch.equal(o, w), turn
    positions.copy_(_positions([[17], [900]]))               # what the graph reads is what the tensors hold
    for graph in graphs:
        graph.replay()
    for o, x in zip(outs, q):
        check(o, cache, x, positions, "bf16")
