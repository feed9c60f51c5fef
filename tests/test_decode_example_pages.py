"""The bookkeeping of the example of a decoding loop, without a GPU: models that only write down which token lies in which slot of their
cache, and a verification that accepts what the test says.  A token must find in its model's own cache every token of the text in front of
it."""
import importlib.util
import pathlib
import types

import numpy as np
import pytest
import torch


@pytest.fixture()
def example(monkeypatch):
    path = pathlib.Path(__file__).resolve().parents[1] / "examples" / "speculative_decode.py"
    spec = importlib.util.spec_from_file_location("speculative_decode_pages", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    monkeypatch.setattr(module, "DEVICE", "cpu")
    return module


class _Model:
    """Slots hold 1 + the token; the cache is [1 layer, 2, pages, 1, page, 1] as a model's."""

    def __init__(self, name, V, known, drafts):
        self.name, self.V, self.dtype, self.known, self.drafts = name, V, torch.float32, known, drafts
        self.furthest = -1

    def cache(self, pages, page):
        return torch.zeros((1, 2, pages, 1, page, 1), dtype=torch.int64)

    def forward(self, tokens, positions, caches, shared_len=None, rows=None):
        cache, = caches
        page, (S, width) = cache.k.shape[2], cache.table.shape
        for s in range(S):
            for t in range(tokens.shape[1]):
                at = int(positions[s, t])
                if at >= 0:
                    assert at < width * page, "%s: position %d lies behind the table" % (self.name, at)
                    cache.k[cache.table[s, at // page], 0, at % page, 0] = 1 + int(tokens[s, t])
        K = S // len(self.known)
        for s in range(S):
            text = self.known[s // K]
            last = int(positions[s].max())
            self.furthest = max(self.furthest, last)
            held = [int(cache.k[cache.table[s, j // page], 0, j % page, 0]) - 1 for j in range(min(last + 1, len(text)))]
            assert held == text[:len(held)], "%s: sequence %d reads %s at %d" % (
                self.name, s, held, next(j for j in range(len(held)) if held[j] != text[j]))
            if shared_len is not None and last >= 0:                                # what a prefix's drafts share lies in the same pages
                whole = int(shared_len[s // K]) // page
                assert torch.equal(cache.table[s, :whole], cache.table[s // K * K, :whole])
        return torch.zeros((S, rows or tokens.shape[1], self.V))


def _decode(example, monkeypatch, accepted, lengths, drafts, length, new, page, V=97, seed=0):
    """`accepted(prompt, iteration)`: how many drafted tokens the verification leaves."""
    rng = np.random.default_rng(seed)
    prompts = [rng.integers(0, V, n).tolist() for n in lengths]
    known = [list(p) for p in prompts]

    def sample(z, u=None, draw=True, kept=None, **kw):
        return torch.from_numpy(rng.integers(0, V, z.shape[0]).astype(np.int32)) if draw else None, kept, None

    def verify(target, draft, tokens, temperature, rng_seed, iteration, pending_state=None):
        B, K, L = tokens.shape
        taken = torch.tensor([accepted(b, iteration) for b in range(B)], dtype=torch.int32)
        by = torch.from_numpy(rng.integers(0, K, B).astype(np.int32))
        out = torch.from_numpy(rng.integers(0, V, (B, L + 1)).astype(np.int32))
        for b in range(B):
            out[b, :taken[b]] = tokens[b, by[b], :taken[b]]
            known[b] += out[b, :taken[b] + 1].tolist()
        return taken, by, out, None

    monkeypatch.setattr(example, "sg", types.SimpleNamespace(
        PagedCache=lambda k, v, table: types.SimpleNamespace(k=k, v=v, table=table), specgbv_sample_filtered=sample,
        specgbv_verify_ex=verify, specgbv_pending_state_bytes=lambda B: 16 * 12 * B))
    models = [_Model(name, V, known, drafts) for name in ("target", "draft")]
    text, iterations = example.decode(*models, prompts, drafts, length, new, page)
    for b, (p, t) in enumerate(zip(prompts, text)):
        assert t == known[b][:len(t)] and len(p) + new <= len(t) <= len(p) + new + length
    return text, iterations


@pytest.mark.parametrize("fast,slow", [(0, 1), (1, 0)])
@pytest.mark.parametrize("drafts,length,page,new", [(4, 8, 16, 64), (1, 4, 8, 40), (3, 5, 8, 33)])
def test_a_prompt_that_is_ahead_of_the_slowest_one(example, monkeypatch, fast, slow, drafts, length, page, new):
    """One prompt takes all but one token a block, the other none: the first is done long before and must not outgrow its table."""
    _decode(example, monkeypatch, lambda b, i: length - 1 if b == fast else 0, [41, 37] if fast == 0 else [5, 60], drafts, length, new, page)


@pytest.mark.parametrize("drafts,length,page,prompt", [(2, 4, 8, 4), (3, 8, 8, 16), (1, 5, 16, 11), (4, 7, 8, 1), (2, 1, 8, 7)])
def test_blocks_that_are_taken_whole_and_end_on_a_page(example, monkeypatch, drafts, length, page, prompt):
    """The draft model has not seen a block's last drafted token when the block is verified: a page that ends with it is not yet whole."""
    assert any((prompt + i * (length + 1) + length) % page == 0 for i in range(page))
    _decode(example, monkeypatch, lambda b, i: length, [prompt, prompt + 3], drafts, length, 8 * page, page)


def test_blocks_that_are_taken_in_part(example, monkeypatch):
    rng = np.random.default_rng(3)
    for length in (1, 3, 8):
        _decode(example, monkeypatch, lambda b, i: int(rng.integers(0, length + 1)), [1, 9, 30, 64], 3, length, 50, 8, seed=length)


@pytest.mark.gpu
@pytest.mark.parametrize("drafts,length,page", [(2, 4, 8), (1, 8, 8), (3, 7, 16)])
def test_a_draft_model_that_is_the_target_is_always_right(drafts, length, page):
    """top_k 1 and one model for both: every drafted token is taken for as long as the draft model's cache holds what the text says.  Rows of one
    token and of a block round differently: where the logits of the two likeliest tokens are within 1e-3, far beyond float32's errors over two
    layers, a block may be cut short."""
    from test_gpu_decode_example import _plain_logits
    path = pathlib.Path(__file__).resolve().parents[1] / "examples" / "speculative_decode.py"
    spec = importlib.util.spec_from_file_location("speculative_decode_same", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    target = module.Model(1, V=500, E=128, D=64, dtype=torch.float32)
    draft = module.Model(2, dtype=torch.float32, V=500, E=128, D=64, like=target, noise=0.0)
    prompts = [np.random.default_rng(n).integers(0, 500, n).tolist() for n in (3, 8, 17)]
    new = 6 * (length + 1)
    text, iterations = module.decode(target, draft, prompts, drafts, length, new=new, page=page, top_k=1, top_p=1.0)
    near = 0
    for p, t in zip(prompts, text):
        best = np.sort(_plain_logits(target, t)[len(p) - 1:-1], axis=-1)[:, -2:]
        near += int((best[:, 1] - best[:, 0] < 1e-3).sum())
    assert near <= 1 and 6 <= iterations <= 6 + near
