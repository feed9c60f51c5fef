"""Block tables on the GPU against lists on the host, over many steps of growing, ending and beginning requests, with and without enough
pages, and the places of new tokens."""
import numpy as np
import pytest

import paper_2604_25925_amd as sg
from pages_util import Pool

pytestmark = pytest.mark.gpu


def _free(pool):
    head, count = pool.ends.tolist()
    ring = pool.ring.tolist()
    return [ring[(head + i) % len(ring)] for i in range(count)]


def _check(pool, host, label):
    B, K = pool.prefixes, pool.drafts
    assert pool.table.view(B, K, -1).tolist() == host.rows, label
    assert [tuple(x) for x in pool.held.tolist()] == host.held, label
    assert _free(pool) == list(host.free), label
    # every page is in one place: free, shared by a request's drafts, or a draft's own
    seen = list(host.free)
    for b in range(B):
        w, h = host.held[b]
        seen += host.rows[b][0][:h]
        for k in range(1, K):
            assert host.rows[b][k][:w] == host.rows[b][0][:w]
            seen += host.rows[b][k][w:h]
    assert len(seen) == len(set(seen)) and min(seen, default=0) >= 0, label


@pytest.mark.parametrize("B,K,width,page,pages", [(1, 1, 4, 8, 4), (1, 8, 40, 16, 200), (3, 2, 9, 8, 30), (32, 8, 20, 16, 2000), (40, 3, 30, 8, 700), (130, 1, 12, 16, 600),
                                                  (1000, 2, 20, 16, 9000), (1025, 1, 10, 8, 4000), (70, 4, 300, 8, 30000), (2500, 1, 30, 8, 20000), (1024, 4, 16, 8, 30000), (1024, 1, 30, 8, 9000), (128, 8, 64, 16, 50000),
                                                  (341, 3, 30, 8, 20000), (342, 3, 30, 8, 20000)])
def test_steps_of_a_batch(B, K, width, page, pages):
    import torch
    gen = np.random.default_rng(B * 10 + K)
    pool = sg.PagePool.empty(B, width, pages, page_size=page, drafts=K)
    order = gen.permutation(pages).astype(np.int32)
    head = int(gen.integers(0, pages))
    pool.ring.copy_(torch.from_numpy(np.roll(order, head)))
    pool.ends[0] = head
    host = Pool(B, K, width, page, order.tolist())
    length, ws = np.zeros(B, int), None
    states = set()
    for step in range(14):
        room = int(gen.choice([0, 1, 5, 17]))
        grown = np.where(length > 0, length + gen.integers(0, 18, B), 0)
        ends, begins = gen.random(B) < 0.1, gen.random(B) < (1.0 if step == 0 else 0.5)
        length = np.where(ends, -int(gen.integers(0, 3)), np.where((length <= 0) & begins, gen.integers(1, width * page + 20, B), grown))
        if step == 9:                                        # some texts get shorter
            length = np.where(gen.random(B) < 0.5, length // 2, length)
        chosen = gen.integers(-1, K + 1, B)
        label = (B, K, width, page, pages, step)
        print("case", label, flush=True)
        shared, served, ws = sg.specgbv_pages_advance(pool, torch.from_numpy(length.astype(np.int32)).cuda(),
                                                      chosen=torch.from_numpy(chosen.astype(np.int32)).cuda() if step % 4 else None, room=room, workspace=ws)
        want = host.advance(length.tolist(), chosen.tolist() if step % 4 else [0] * B, room)
        assert (shared.tolist(), served.tolist()) == (want[0], want[1]), label
        _check(pool, host, label)
        states |= set(served.tolist())
        length = np.where(np.array(want[1]) == 1, length, [host.held[b][0] * page for b in range(B)])
    if B > 2:
        assert states >= {1, -1}
    # everything ends: all pages are free again
    shared, served, _ = sg.specgbv_pages_advance(pool, torch.zeros(B, dtype=torch.int32, device="cuda"), workspace=ws)
    host.advance([0] * B, [0] * B, 0)
    _check(pool, host, "end")
    assert sorted(_free(pool)) == list(range(pages)) and (pool.table == -1).all()


def test_requests_that_do_not_fit_keep_what_they_have():
    import torch
    pool = sg.PagePool.empty(4, 8, 10, page_size=8, drafts=2)
    length = torch.tensor([20, 30, 1, 64], dtype=torch.int32, device="cuda")
    shared, served, _ = sg.specgbv_pages_advance(pool, length, room=1)
    # 2 + 2 pages, 3 + 2 pages, 2 pages (one too many), longer than the table
    assert served.tolist() == [1, 1, 0, -1] and shared.tolist() == [16, 24, 0, 0]
    assert pool.ends.tolist() == [9, 1] and pool.held.tolist() == [[2, 3], [3, 4], [0, 0], [0, 0]]
    assert (pool.table[4:] == -1).all()
    length[1] = 0
    shared, served, _ = sg.specgbv_pages_advance(pool, length, room=1)
    assert served.tolist() == [1, 1, 1, -1] and pool.ends.tolist() == [1, 4]      # what request 1 gave back came behind the last free page
    assert pool.table[4, 0].item() == 9 and pool.table[5, 0].item() == 4


def test_extremes_and_states_out_of_range():
    """Numbers that no loop makes: nothing is read or written out of range, whatever comes of them."""
    import torch
    big = 2 ** 31 - 1
    for B, K, width in ((3, 2, 5), (1500, 2, 30)):
        pool = sg.PagePool.empty(B, width, 50, page_size=8, drafts=K)
        length = torch.full((B,), big, dtype=torch.int32, device="cuda")
        shared, served, ws = sg.specgbv_pages_advance(pool, length, room=big)
        assert (served == -1).all() and (shared == 0).all() and (pool.table == -1).all()
        guard = torch.full((B * K + 2, width + 3), 77, dtype=torch.int32, device="cuda")
        inner = guard[1:-1, :width]
        inner.fill_(-1)
        strange = sg.PagePool(inner, pool.ring, torch.tensor([-5, big], dtype=torch.int32, device="cuda"),
                              torch.tensor([[big, -3], [-7, big], [4, 2]] * (B // 3), dtype=torch.int32, device="cuda"), drafts=K, page_size=8)
        for step in range(3):
            sg.specgbv_pages_advance(strange, torch.from_numpy(np.random.default_rng(step).integers(-9, 60, B).astype(np.int32)).cuda(), room=3, workspace=ws)
        torch.cuda.synchronize()
        assert (guard[0] == 77).all() and (guard[-1] == 77).all() and (guard[:, width:] == 77).all()
        assert 0 <= strange.ends[0].item() < 50 and 0 <= strange.ends[1].item() <= 50


def test_pages_in_a_captured_graph_and_on_another_stream():
    import torch
    for B, width in ((6, 20), (300, 300)):
        pools = [sg.PagePool.empty(B, width, B * width // 2, page_size=8, drafts=2) for _ in range(2)]
        length = torch.zeros(B, dtype=torch.int32, device="cuda")
        shared, served, ws = sg.specgbv_pages_advance(pools[0], length, room=9)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            sg.specgbv_pages_advance(pools[0], length, room=9, shared_len=shared, served=served, workspace=ws)
        gen = np.random.default_rng(B)
        side = torch.cuda.Stream()
        for turn in range(5):
            length.copy_(torch.from_numpy(gen.integers(-3, width * 4, B).astype(np.int32)))
            graph.replay()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                want = sg.specgbv_pages_advance(pools[1], length, room=9)
            torch.cuda.synchronize()
            assert torch.equal(want[0], shared) and torch.equal(want[1], served)
            for x in ("table", "ring", "ends", "held"):
                assert torch.equal(getattr(pools[0], x), getattr(pools[1], x)), (turn, x)


@pytest.mark.parametrize("B,K,T,page,width", [(1, 1, 1, 8, 1), (3, 2, 7, 8, 6), (32, 8, 24, 16, 130), (5, 1, 400, 64, 9), (1, 1, 5000, 16, 20)])
def test_slot_maps(B, K, T, page, width):
    import torch
    gen = np.random.default_rng(B + T)
    S, pages = B * K, B * K * width + 3
    table = gen.permutation(pages)[:S * width].astype(np.int32).reshape(S, width)
    table[gen.random(table.shape) < 0.1] = gen.choice([-1, pages, -2 ** 31, 2 ** 31 - 1])
    start = gen.integers(-3, width * page + 5, B).astype(np.int32)
    count = gen.integers(-2, T + 3, B).astype(np.int32)
    start[-1] = 2 ** 31 - 2
    dev = [torch.from_numpy(x).cuda() for x in (table, start, count)]
    for right in (False, True):
        want_p, want_s = np.full((S, T), -1, np.int64), np.full((S, T), -1, np.int64)
        for s in range(S):
            n = min(max(int(count[s // K]), 0), T)
            for i in range(n):
                p = int(start[s // K]) + i
                if not 0 <= p < 2 ** 31:
                    continue
                t = T - n + i if right else i
                want_p[s, t] = p
                if p // page < width and 0 <= table[s, p // page] < pages:
                    want_s[s, t] = int(table[s, p // page]) * page + p % page
        positions, slots = sg.specgbv_slot_map(*dev, T, page_size=page, pages=pages, drafts=K, right=right)
        assert positions.dtype is torch.int32 and slots.dtype is torch.int64
        assert (positions.cpu().numpy() == want_p).all() and (slots.cpu().numpy() == want_s).all()
        alone, none = sg.specgbv_slot_map(*dev, T, page_size=page, pages=pages, drafts=K, right=right, flat=False)
        assert none is None and torch.equal(alone, positions)
        room = [torch.full((S, T + 5), 9, dtype=d, device="cuda") for d in (torch.int32, torch.int64)]
        sg.specgbv_slot_map(*dev, T, page_size=page, pages=pages, drafts=K, right=right, positions=room[0][:, 1:T + 1], slots=room[1][:, 2:T + 2])
        assert torch.equal(room[0][:, 1:T + 1], positions) and torch.equal(room[1][:, 2:T + 2], slots)
        assert (room[0][:, T + 1:] == 9).all() and (room[1][:, T + 2:] == 9).all() and (room[0][:, 0] == 9).all()


def test_slots_beyond_31_bits():
    import torch
    table = torch.tensor([[2 ** 30 - 1]], dtype=torch.int32, device="cuda")
    one = torch.tensor([5], dtype=torch.int32, device="cuda")
    _, slots = sg.specgbv_slot_map(table, one, one, 5, page_size=64, pages=2 ** 30)
    assert slots.tolist() == [[(2 ** 30 - 1) * 64 + 5 + i for i in range(5)]]
