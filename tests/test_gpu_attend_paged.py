"""specgbv_attend_paged against the definition in float64, query by query (needs an MI355X: run with -m gpu).  The bounds are those of
decoding_util.attend_bound."""
import numpy as np
import pytest

from decoding_util import check_attend, host, make_cache, plain_attend, torch_dtype

pytestmark = pytest.mark.gpu


def _inputs(S, T, H, G, D, page, dtype, width, seed=0, token_major=False, scale=1.5, fill=None):
    import torch
    rng = np.random.default_rng(seed + 31 * D + 7 * T + S)
    k, v, table = make_cache(rng, S, width, page, G, D, dtype, token_major, fill=fill)
    q = torch.from_numpy(rng.normal(0, scale, (S, T, H, D)).astype(np.float32)).cuda().to(torch_dtype(dtype))
    return rng, q, k, v, table


def _run(S, T, H, G, D, page, dtype, width, window=0, seed=0, token_major=False, positions=None, max_len=None, **kw):
    import torch
    import paper_2604_25925_amd as sg
    rng, q, k, v, table = _inputs(S, T, H, G, D, page, dtype, width, seed, token_major)
    if positions is None:
        last = rng.integers(0, width * page, (S, 1))
        last[0] = width * page - 1
        positions = np.maximum(last - T + 1 + np.arange(T), -1)
    pos = torch.from_numpy(np.asarray(positions, np.int32)).cuda()
    out, ws = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, pos, window=window, max_len=max_len, **kw)
    torch.cuda.synchronize()
    check_attend(out, q, k, v, table, pos, dtype, window, label=str((S, T, H, G, D, page, dtype, width, window)))
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [8, 40, 64, 72, 80, 96, 128, 136, 192, 256])
def test_head_dimensions(dtype, D):
    _run(2, 1, 4, 2, D, 16, dtype, 9)
    _run(2, 3, 6, 1, D, 8, dtype, 21, token_major=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G", [(1, 1), (8, 8), (5, 1), (14, 2), (16, 1), (21, 3), (64, 2)])
def test_groups_of_heads(dtype, H, G):
    _run(2, 1, H, G, 64, 32, dtype, 5)
    _run(1, 9, H, G, 64, 32, dtype, 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [8, 16, 24, 40, 128])
def test_page_sizes(dtype, page):
    _run(3, 2, 4, 2, 128, page, dtype, 1 + 300 // page)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_short_length(dtype):
    """Sequences of 0 to 70 tokens, one query each: the tile's end in every place, and none at all."""
    n = 71
    _run(n, 1, 4, 2, 64, 8, dtype, 9, positions=np.arange(n)[:, None] - 1)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64), ("bf16", 256), ("f32", 128), ("f32", 256)])
@pytest.mark.parametrize("T,H", [(17, 4), (40, 8), (130, 2)])
def test_many_queries(dtype, D, T, H):
    _run(2, T, H, 2, D, 16, dtype, 12)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 100, 1000])
def test_windows(dtype, window):
    _run(3, 5, 4, 2, 64, 16, dtype, 20, window=window)


def test_padding_and_positions_out_of_order():
    pos = [[-1, 5, 300, -7], [0, 0, 299, 12], [-1, -1, -1, -1], [40, 39, 38, 2 ** 31 - 1]]
    _run(4, 4, 6, 2, 128, 16, "bf16", 20, positions=pos)
    _run(4, 4, 6, 2, 128, 16, "bf16", 20, positions=pos, window=37)
    _run(4, 4, 6, 2, 64, 16, "f32", 20, positions=pos, window=1)


@pytest.mark.parametrize("dtype,S,T,H,G,D,width,window", [("bf16", 1, 1, 8, 2, 128, 700, 0), ("bf16", 3, 2, 4, 4, 64, 300, 0), ("f32", 1, 1, 4, 1, 64, 500, 0),
                                                          ("bf16", 2, 5, 4, 1, 80, 400, 3000), ("bf16", 1, 1, 2, 1, 256, 300, 0)])
def test_long_contexts_are_split(dtype, S, T, H, G, D, width, window):
    import paper_2604_25925_amd as sg
    _run(S, T, H, G, D, 16, dtype, width, window=window)
    rng, q, k, v, table = _inputs(S, T, H, G, D, 16, dtype, width)
    assert sg.specgbv_attend_workspace_bytes(sg.PagedCache(k, v, table), q, window=window) > 0
    # the hint is a hint: sequences that reach further, or not as far
    for max_len in (1, 600, 1 << 29):
        _run(S, T, H, G, D, 16, dtype, width, window=window, max_len=max_len)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,K,T,H,G,D,page", [(2, 8, 1, 8, 2, 128, 16), (3, 4, 1, 4, 1, 64, 32), (2, 2, 9, 8, 2, 128, 16), (1, 3, 5, 14, 2, 64, 8),
                                              (2, 8, 9, 8, 2, 64, 64), (1, 5, 3, 2, 1, 256, 16)])
@pytest.mark.parametrize("window", [0, 150])
def test_drafts_that_share_their_prefix(dtype, B, K, T, H, G, D, page, window):
    import torch
    import paper_2604_25925_amd as sg
    rng = np.random.default_rng(K * 100 + T)
    width = 1 + 480 // page
    length = rng.integers(0, width * page - 20 - T, (B, 1))
    length[0] = width * page - 20 - T
    if B > 2:
        length[2] = page - 1                                 # no whole page
    whole = length // page
    S = B * K
    table = rng.permutation(S * width).astype(np.int32).reshape(B, K, width)
    table = np.where(np.arange(width) < whole[:, :, None], table[:, :1], table).reshape(S, width)
    k, v, _ = make_cache(rng, S, width, page, G, D, dtype)
    q = torch.from_numpy(rng.normal(0, 1.5, (S, T, H, D)).astype(np.float32)).cuda().to(torch_dtype(dtype))
    pos = np.repeat(length + rng.integers(0, 8, (B, 1)), K, axis=0) + np.arange(T)
    pos[S - 1, 0] = -1
    pos, table = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(table).cuda()
    cache = sg.PagedCache(k, v, table)
    for shared in (whole * page, whole * 0, np.maximum(whole * page - 5, 0)):      # also fewer tokens than are shared
        sl = torch.from_numpy(shared.reshape(B).astype(np.int32)).cuda()
        out, ws = sg.specgbv_attend_paged(cache, q, pos, window=window, shared_len=sl)
        ws.fill_(255)                                        # (numbers that are none: what is joined was written by the call)
        out, _ = sg.specgbv_attend_paged(cache, q, pos, window=window, shared_len=sl, workspace=ws, out=out)
        torch.cuda.synchronize()
        check_attend(out, q, k, v, table, pos, dtype, window, label="shared")


def test_wild_shared_lengths_stay_inside():
    """A statement that does not hold gives another result, not a read outside the cache."""
    import torch
    import paper_2604_25925_amd as sg
    rng, q, k, v, table = _inputs(4, 1, 4, 2, 64, 16, "bf16", 6)
    pos = torch.full((4, 1), 60, dtype=torch.int32, device="cuda")
    sl = torch.tensor([2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    out, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, pos, shared_len=sl)
    assert bool(torch.isfinite(out.float()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_are_not_there(dtype):
    import torch
    import paper_2604_25925_amd as sg
    rng, q, k, v, table = _inputs(4, 3, 4, 2, 64, 16, dtype, 10)
    table[0, 0], table[0, 4], table[1, 9], table[2, 1] = -1, k.shape[0], 2 ** 31 - 1, -2 ** 31
    table[3] = -1                                            # none at all
    pos = torch.tensor([[5, 70, 159], [159, 10 ** 6, 2 ** 31 - 1], [15, 16, 17], [0, 50, 100]], dtype=torch.int32, device="cuda")
    for window in (0, 20):
        out, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, pos, window=window)
        torch.cuda.synchronize()
        check_attend(out, q, k, v, table, pos, dtype, window)
        assert bool((out[3] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_what_a_query_does_not_see_does_not_enter(dtype, value):
    """Slots behind the last token, tokens that only later queries see and tokens in front of the window hold numbers that are
    none: the results are those of a cache that holds zeros there, and queries that do see them are not finite."""
    import torch
    import paper_2604_25925_amd as sg
    S, T, H, G, D, page, width = 3, 4, 4, 2, 64, 16, 8
    rng, q, k, v, table = _inputs(S, T, H, G, D, page, dtype, width)
    pos = np.array([[20, 21, 22, 23], [99, 100, 101, 102], [0, 1, 2, 3]], np.int32)
    for window in (0, 30):
        k1, v1 = k.clone(), v.clone()
        for s in range(S):
            at = np.arange(width * page)
            bad = at >= pos[s, 2]                            # the last two queries' own tokens, and everything behind them
            if window:
                bad |= at <= pos[s, 0] - window
            for a in at[bad]:
                k1[table[s, a // page], :, a % page] = value
                v1[table[s, a // page], :, a % page, ::3] = value
        p = torch.from_numpy(pos).cuda()
        out, _ = sg.specgbv_attend_paged(sg.PagedCache(k1, v1, table), q, p, window=window)
        torch.cuda.synchronize()
        ref, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, p, window=window)
        assert torch.equal(out[:, :2], ref[:, :2])
        check_attend(out[:, :2], q[:, :2], k, v, table, p[:, :2], dtype, window)
        if not window:
            k1 = k.clone()                                   # keys in order, one value that is none: the entries it reaches
            out, _ = sg.specgbv_attend_paged(sg.PagedCache(k1, v1, table), q, p)
            bad = ~np.isfinite(host(out[:, 2:]))
            assert bad[..., ::3].all() and not bad[..., 1::3].any() and not bad[..., 2::3].any()
            assert np.isfinite(host(out[:, :2])).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_the_types_lowest_value(dtype):
    """Keys that give scores of about -1e38 and of -inf next to ordinary ones, and sequences that hold such keys alone."""
    import torch
    import paper_2604_25925_amd as sg
    S, H, G, D, page, width = 3, 2, 1, 64, 16, 6
    rng, q, k, v, table = _inputs(S, 1, H, G, D, page, dtype, width)
    q.zero_()
    q[..., 0] = 1.0
    at = np.arange(90)
    for s in range(S):
        for a in at:
            k[table[s, a // page], 0, a % page, 0] = -3.0e38 if s == 1 or a % 3 == 0 else (float("-inf") if a % 3 == 1 and s == 0 else float(rng.normal()))
    pos = torch.full((S, 1), 89, dtype=torch.int32, device="cuda")
    out, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, pos, scale=0.25)
    torch.cuda.synchronize()
    check_attend(out, q, k, v, table, pos, dtype, scale=0.25)


def test_rising_and_falling_scores():
    """Scores that rise by hundreds along the sequence (the reference is raised again and again), and that fall."""
    import torch
    import paper_2604_25925_amd as sg
    S, H, G, D, page, width = 2, 2, 1, 64, 16, 40
    for dtype in ("bf16", "f32"):
        rng, q, k, v, table = _inputs(S, 1, H, G, D, page, dtype, width)
        q.zero_()
        q[..., 0] = 8.0
        for s in range(S):
            ramp = np.linspace(-500, 500, width * page) * (1 if s == 0 else -1)
            for a in range(width * page):
                k[table[s, a // page], 0, a % page, 0] = float(ramp[a])
        pos = torch.full((S, 1), width * page - 1, dtype=torch.int32, device="cuda")
        out, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, pos)
        torch.cuda.synchronize()
        check_attend(out, q, k, v, table, pos, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_of_queries_and_output(dtype):
    import torch
    import paper_2604_25925_amd as sg
    S, T, H, G, D, page, width = 3, 2, 4, 2, 64, 16, 5
    rng, q, k, v, table = _inputs(S, T, H, G, D, page, dtype, width)
    cache = sg.PagedCache(k, v, torch.cat((table, table), dim=1)[:, :width])        # rows of the table further apart
    pos = torch.tensor([[40, 41, 7], [70, 71, 7], [0, 1, 7]], dtype=torch.int32, device="cuda")[:, :2]
    ref, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, pos.contiguous())
    for shift in (1, 2, 8):
        wide = torch.zeros((S, T, H + 3, D + shift), dtype=q.dtype, device="cuda")
        view = wide[:, :, 1:1 + H, shift:]
        view.copy_(q)
        into = torch.full((S, H, T, D + shift), 7.0, dtype=q.dtype, device="cuda")
        out = into[..., shift:].transpose(1, 2)
        sg.specgbv_attend_paged(cache, view, pos, out=out)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
        assert bool((into[..., :shift] == 7).all())


def test_caches_beyond_32_bit_offsets():
    import torch
    import paper_2604_25925_amd as sg
    pages, G, page, D = 1100, 8, 1024, 256
    k = torch.zeros((pages, G, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    k[pages - 2:].normal_()
    v[pages - 2:].normal_()
    q = torch.randn((1, 1, G, D), device="cuda").bfloat16()
    pos = torch.tensor([[1100]], dtype=torch.int32, device="cuda")
    out, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, pos)
    small = sg.PagedCache(k[pages - 2:], v[pages - 2:], torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    ref, _ = sg.specgbv_attend_paged(small, q, pos)
    assert torch.equal(out, ref)
    check_attend(out, q, small.k, small.v, small.table, pos, "bf16")


def test_results_do_not_change_from_call_to_call():
    import torch
    import paper_2604_25925_amd as sg
    rng, q, k, v, table = _inputs(2, 2, 8, 2, 128, 16, "bf16", 300)
    cache = sg.PagedCache(k, v, table)
    pos = torch.tensor([[4000, 4001], [2500, 2501]], dtype=torch.int32, device="cuda")
    ref, ws = sg.specgbv_attend_paged(cache, q, pos)
    for _ in range(10):
        ws.random_(0, 256)
        out, _ = sg.specgbv_attend_paged(cache, q, pos, workspace=ws)
        assert torch.equal(out, ref)


def test_replays_of_a_captured_call():
    import torch
    import paper_2604_25925_amd as sg
    rng, q, k, v, table = _inputs(4, 1, 8, 2, 128, 16, "bf16", 60)
    sl = torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    table[1, :30], table[3, :30] = table[0, :30].clone(), table[2, :30].clone()
    cache = sg.PagedCache(k, v, table)
    pos = torch.full((4, 1), 900, dtype=torch.int32, device="cuda")
    out, ws = sg.specgbv_attend_paged(cache, q, pos, shared_len=sl)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sg.specgbv_attend_paged(cache, q, pos, shared_len=sl, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sg.specgbv_attend_paged(cache, q, pos, shared_len=sl, out=out, workspace=ws)
    for step in range(5):
        q.normal_()
        pos.fill_(100 * step + 60)
        sl.fill_(min(30 * 16, (100 * step + 60) // 16 * 16))
        eager, _ = sg.specgbv_attend_paged(cache, q, pos, shared_len=sl)
        ws.fill_(step)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        check_attend(out, q, k, v, table, pos, "bf16")


@pytest.mark.parametrize("dtype,S,T,width,window", [("bf16", 70, 1, 260, 0), ("f32", 66, 2, 150, 0), ("bf16", 65, 9, 160, 700)])
def test_more_sequences_than_lanes(dtype, S, T, width, window):
    """Units beyond 64 are cut alike, whatever their lengths; some are empty."""
    import paper_2604_25925_amd as sg
    rng = np.random.default_rng(S)
    last = rng.integers(-1, width * 16, (S, 1))
    last[1], last[2], last[S - 1] = -1, 0, width * 16 - 1
    positions = np.maximum(last - T + 1 + np.arange(T), -1)
    _run(S, T, 4, 1, 64, 16, dtype, width, window=window, positions=positions)
    rng, q, k, v, table = _inputs(S, T, 4, 1, 64, 16, dtype, width)
    assert sg.specgbv_attend_workspace_bytes(sg.PagedCache(k, v, table), q, window=window) > 0


@pytest.mark.parametrize("dtype,B,K,T,H,G", [("bf16", 70, 2, 1, 4, 1), ("f32", 66, 3, 2, 2, 1), ("bf16", 65, 4, 9, 4, 2)])
def test_more_prefixes_than_lanes(dtype, B, K, T, H, G):
    import torch
    import paper_2604_25925_amd as sg
    rng = np.random.default_rng(B * K)
    page, width, D = 16, 40, 64
    length = rng.integers(0, width * page - T - 8, (B, 1))
    length[0], length[1], length[B - 1] = 0, 5, width * page - T - 8
    whole, S = length // page, B * K
    table = rng.permutation(S * width).astype(np.int32).reshape(B, K, width)
    table = np.where(np.arange(width) < whole[:, :, None], table[:, :1], table).reshape(S, width)
    k, v, _ = make_cache(rng, S, width, page, G, D, dtype)
    q = torch.from_numpy(rng.normal(0, 1.5, (S, T, H, D)).astype(np.float32)).cuda().to(torch_dtype(dtype))
    pos = np.repeat(length, K, axis=0) + np.arange(T) + rng.integers(0, 8, (S, 1))
    pos, table = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(table).cuda()
    sl = torch.from_numpy((whole * page).reshape(B).astype(np.int32)).cuda()
    cache = sg.PagedCache(k, v, table)
    out, ws = sg.specgbv_attend_paged(cache, q, pos, shared_len=sl)
    ws.fill_(255)
    out, _ = sg.specgbv_attend_paged(cache, q, pos, shared_len=sl, workspace=ws)
    torch.cuda.synchronize()
    check_attend(out, q, k, v, table, pos, dtype, label="shared")


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 200)])
def test_many_parts_are_joined(dtype, D):
    """One sequence over the whole card, and one that is empty next to it: dozens of parts a row."""
    _run(2, 1, 2, 1, D, 16, dtype, 1500, positions=[[23999], [-1]])
    _run(1, 3, 5, 1, D, 16, dtype, 1100, positions=[[12, 17000, 17599]])


@pytest.mark.parametrize("dtype,B,K,T,H,G,D,page", [("bf16", 2, 8, 1, 8, 2, 128, 16), ("f32", 2, 4, 1, 4, 1, 64, 32), ("bf16", 2, 2, 9, 8, 2, 128, 16),
                                                    ("f32", 1, 3, 5, 14, 2, 64, 8), ("bf16", 2, 8, 9, 8, 2, 64, 64), ("f32", 1, 8, 9, 4, 1, 128, 16),
                                                    ("bf16", 1, 5, 3, 2, 1, 256, 16), ("bf16", 1, 20, 9, 1, 1, 64, 8)])
@pytest.mark.parametrize("window", [0, 1150])
def test_drafts_that_share_long_prefixes(dtype, B, K, T, H, G, D, page, window):
    """Beyond the lengths up to which drafts are taken by themselves: drafts of positions of their own, some without tokens of
    their own, fewer tokens stated than are shared, pages that are not there."""
    import torch
    import paper_2604_25925_amd as sg
    rng = np.random.default_rng(K * 100 + T)
    width = 1 + 1400 // page
    length = np.full((B, 1), width * page - 20 - T)
    length[1:] = rng.integers(0, width * page - 20 - T, (B - 1, 1))
    whole, S = length // page, B * K
    table = rng.permutation(S * width).astype(np.int32).reshape(B, K, width)
    table = np.where(np.arange(width) < whole[:, :, None], table[:, :1], table).reshape(S, width)
    k, v, _ = make_cache(rng, S, width, page, G, D, dtype)
    q = torch.from_numpy(rng.normal(0, 1.5, (S, T, H, D)).astype(np.float32)).cuda().to(torch_dtype(dtype))
    pos = np.repeat(length, K, axis=0) + np.arange(T) + rng.integers(-3, 8, (S, 1))
    pos[S - 1, 0], pos[0] = -1, whole[0] * page - T + np.arange(T)                 # (draft 0: nothing of its own)
    pos, table = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(table).cuda()
    cache = sg.PagedCache(k, v, table)
    for shared in (whole * page, whole * 0, np.maximum(whole * page - 5, 0)):
        sl = torch.from_numpy(shared.reshape(B).astype(np.int32)).cuda()
        out, ws = sg.specgbv_attend_paged(cache, q, pos, window=window, shared_len=sl)
        ws.fill_(255)
        out, _ = sg.specgbv_attend_paged(cache, q, pos, window=window, shared_len=sl, workspace=ws, out=out)
        torch.cuda.synchronize()
        check_attend(out, q, k, v, table, pos, dtype, window, label="shared")
        near, _ = sg.specgbv_attend_paged(cache, q, pos, window=window, shared_len=sl, max_len=900, workspace=ws)      # taken by themselves
        torch.cuda.synchronize()
        check_attend(near, q, k, v, table, pos, dtype, window, label="alone")
    own = int(whole[0, 0])                                   # a page that no draft shares; page 3 is gone for all
    table[:K, 3], table[0, own], table[K - 1, own] = -1, k.shape[0], -5
    out, _ = sg.specgbv_attend_paged(cache, q, pos, window=window, shared_len=sl, workspace=ws)
    torch.cuda.synchronize()
    check_attend(out, q, k, v, table, pos, dtype, window, label="pages")


@pytest.mark.parametrize("dtype,S,T,H,G,D,page,window", [("bf16", 300, 1, 4, 2, 128, 16, 0), ("f32", 300, 1, 4, 2, 64, 8, 0), ("bf16", 150, 3, 12, 4, 64, 16, 0),
                                                         ("f32", 130, 2, 16, 4, 128, 32, 20), ("bf16", 260, 1, 3, 1, 256, 16, 30), ("f32", 260, 1, 2, 1, 200, 8, 0),
                                                         ("bf16", 90, 9, 24, 6, 80, 16, 0), ("f32", 65, 4, 64, 8, 72, 24, 0)])
def test_many_short_sequences(dtype, S, T, H, G, D, page, window):
    """More units than the card holds at once, of 0 to 200 tokens: each wave by itself.  Queries see nothing, a part of a tile, tiles with
    pages that are not there and numbers that are none behind their positions."""
    import torch
    import paper_2604_25925_amd as sg
    width = -(-200 // page)
    rng, q, k, v, table = _inputs(S, T, H, G, D, page, dtype, width)
    last = rng.integers(-1, width * page, (S, 1))
    last[0], last[1], last[S - 1] = width * page - 1, -1, 0
    pos = np.maximum(last - T + 1 + np.arange(T), -1).astype(np.int32)
    table[5, 1], table[6, 0], table[7] = -1, k.shape[0], -3
    p = torch.from_numpy(pos).cuda()
    cache = sg.PagedCache(k, v, table)
    out, _ = sg.specgbv_attend_paged(cache, q, p, window=window)
    torch.cuda.synchronize()
    check_attend(out, q, k, v, table, p, dtype, window)
    k1, v1 = k.clone(), v.clone()
    for s in range(8, 40):                                   # slots behind the last position
        for a in range(int(pos[s].max()) + 1, width * page):
            k1[table[s, a // page], :, a % page] = float("nan")
            v1[table[s, a // page], :, a % page] = float("inf")
    got, _ = sg.specgbv_attend_paged(sg.PagedCache(k1, v1, table), q, p, window=window)
    torch.cuda.synchronize()
    assert torch.equal(got, out)


@pytest.mark.parametrize("dtype,D", [("bf16", 40), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 96), ("f32", 128), ("f32", 256)])
@pytest.mark.parametrize("T,H,G,width,window", [(33, 8, 1, 12, 0), (70, 4, 1, 13, 50), (150, 4, 2, 40, 0), (40, 7, 1, 150, 0)])
def test_more_rows_than_waves_share(dtype, D, T, H, G, width, window):
    """Queries times heads of a group beyond 256: in one pass and in parts, with and without a window, a ragged last workgroup."""
    _run(2, T, H, G, D, 16, dtype, width, window=window, token_major=D == 64)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("bf16", 256)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_many_rows_and_what_they_do_not_see(dtype, D, value):
    """As for few rows: later queries' tokens, what lies in front of the window and behind the last position hold numbers that are
    none; queries that see such a value get it in its entries alone.  Pages that are not there."""
    import torch
    import paper_2604_25925_amd as sg
    S, T, H, G, page, width = 2, 72, 4, 1, 16, 16
    rng, q, k, v, table = _inputs(S, T, H, G, D, page, dtype, width)
    table[1, 2] = -1
    pos = np.stack([100 + np.arange(T), 20 + np.arange(T)]).astype(np.int32)
    p = torch.from_numpy(pos).cuda()
    for window in (0, 90):
        k1, v1 = k.clone(), v.clone()
        for s in range(S):
            for a in range(width * page):
                if (a > pos[s, T // 2] or (window and a <= pos[s, 0] - window)) and table[s, a // page] >= 0:
                    k1[table[s, a // page], :, a % page] = value
                    v1[table[s, a // page], :, a % page, ::3] = value
        ref, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, p, window=window)
        out, _ = sg.specgbv_attend_paged(sg.PagedCache(k1, v1, table), q, p, window=window)
        torch.cuda.synchronize()
        check_attend(ref, q, k, v, table, p, dtype, window)
        n = T // 2 + 1
        assert torch.equal(out[:, :n], ref[:, :n])
        if not window:
            out, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v1, table), q, p)
            got = host(out)
            assert np.isfinite(got[:, :n]).all() and np.isfinite(got[:, n:, :, 1::3]).all() and np.isfinite(got[:, n:, :, 2::3]).all()
            assert not np.isfinite(got[:, n:, :, ::3]).any()
