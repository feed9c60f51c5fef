"""The example's two loops, tables on the host and tables on the GPU, write the same texts; what a program does between them and specgbv_pages_advance."""
import numpy as np
import pytest

import paper_2604_25925_amd as sg
from test_gpu_decode_example import _plain_logits, _prompts, example  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("drafts,length,page", [(1, 4, 8), (2, 8, 8), (3, 5, 16), (4, 8, 8)])
def test_tables_on_the_host_and_on_the_gpu_give_the_same_text(example, drafts, length, page):  # noqa: F811
    """Over the same caches of float32, the likeliest tokens: token by token, up to one where the target's two likeliest logits are 1e-3 near (from there on the loops may
    write different texts, as their products are of different lengths)."""
    import torch
    target = example.Model(1, V=500, E=128, D=64, dtype=torch.float32)
    draft = example.Model(2, dtype=torch.float32, V=500, E=128, D=64, like=target, noise=0.7)
    prompts = _prompts(500, (3, 8, 41))
    one, turns_one = example.decode(target, draft, prompts, drafts, length, new=24, page=page, top_k=1, top_p=1.0)
    two, turns_two, _ = example.decode_on_gpu(target, draft, prompts, drafts, length, new=24, page=page, top_k=1, top_p=1.0, packed=False)
    apart = 0
    for p, a, b in zip(prompts, one, two):
        if a == b:
            continue
        apart += 1
        n = next((i for i, (x, y) in enumerate(zip(a, b)) if x != y), None)
        assert n is not None, "one text is the beginning of the other"
        best = np.sort(_plain_logits(target, a[:n])[-1])[-2:]
        assert best[1] - best[0] < 1e-3, (n, a[n], b[n])
    if not apart:
        assert turns_one == turns_two


def test_an_unserved_request_has_not_adopted_its_chosen_draft():
    """Two requests of two drafts; the second finds no pages and keeps its own, its drafts' own ones too: given the same chosen draft again once there are pages, it is served as if
    nothing had been in between.  And of the last page, partly filled, each draft has its own: only the chosen one's holds the tokens that stay."""
    import torch

    def numbers(*x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    pool = sg.PagePool.empty(2, 8, 13, page_size=8, drafts=2)
    shared, served, ws = sg.specgbv_pages_advance(pool, numbers(9, 9), room=7)             # 1 shared, 1 of each draft's own: 3 a request
    assert served.tolist() == [1, 1] and shared.tolist() == [8, 8] and pool.ends.tolist()[1] == 7
    rows = pool.table.view(2, 2, 8).clone()
    assert not torch.equal(rows[:, 0, 1], rows[:, 1, 1])
    # each wants seven pages more than it has: they are there for the first alone
    shared, served, ws = sg.specgbv_pages_advance(pool, numbers(17, 17), chosen=numbers(1, 1), room=30, workspace=ws)
    assert served.tolist() == [1, 0] and shared.tolist() == [16, 8]
    assert torch.equal(pool.table.view(2, 2, 8)[1], rows[1]) and pool.held.tolist()[1] == [1, 2]
    assert (pool.table.view(2, 2, 8)[0, :, 1] == rows[0, 1, 1]).all()                       # adopted by both drafts
    sg.specgbv_pages_advance(pool, numbers(0, 17), chosen=numbers(0, 1), room=30, workspace=ws)
    after = pool.table.view(2, 2, 8)
    assert (after[1, :, 1] == rows[1, 1, 1]).all() and pool.held.tolist() == [[0, 0], [2, 6]]
    assert not torch.equal(after[1, 0, 2:6], after[1, 1, 2:6])
