"""The example's loop on the GPU: block tables, positions, append, attention, truncated sampling and verification together, over caches of 16 or 32
bits and of 4 (needs an MI355X: run with -m gpu)."""
import numpy as np
import pytest

import packed_util
from test_gpu_decode_example import _plain_logits, _prompts, example  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def _models(example, dtype, noise=0.7, V=500):
    target = example.Model(1, V=V, E=128, D=64, dtype=dtype)
    return target, example.Model(2, dtype=dtype, V=V, E=128, D=64, like=target, noise=noise)


def _all_free(pool):
    import torch
    head, count = pool.ends.tolist()
    assert count == pool.pages and sorted(pool.ring.tolist()) == list(range(pool.pages))
    assert (pool.table == -1).all() and not torch.any(pool.held)


@pytest.mark.parametrize("drafts,length,page", [(1, 4, 8), (3, 5, 16), (4, 8, 8)])
def test_the_likeliest_tokens_are_those_of_the_target_alone(example, drafts, length, page):  # noqa: F811
    """As for the loop that keeps its tables on the host."""
    import torch
    target, draft = _models(example, torch.float32)
    prompts = _prompts(500, (3, 8, 41))
    text, iterations, pool = example.decode_on_gpu(target, draft, prompts, drafts, length, new=24, page=page, top_k=1, top_p=1.0, packed=False)
    assert 24 / (length + 1) <= iterations < 24
    _all_free(pool)
    for p, t in zip(prompts, text):
        assert t[:len(p)] == p and len(t) >= len(p) + 24
        z = _plain_logits(target, t)
        for i in range(len(p) - 1, len(t) - 1):
            best = np.sort(z[i])[-2:]
            assert t[i + 1] == int(z[i].argmax()) or best[1] - best[0] < 1e-3


def _held_logits(m, text):
    """Logits [tokens, V] of a text in float64 on the CPU, its keys and values rounded as the cache holds them."""
    import math

    def f(w):
        return w.detach().double().cpu().numpy()

    def norm(x):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)

    def held(x):
        return packed_util.values(*packed_util.quantise(x))

    n, D, H, G = len(text), m.D, m.heads, m.kv_heads
    x = f(m.embed)[np.asarray(text)]
    angle = np.arange(n)[:, None] * f(m.inv_freq)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    for w in m.layers:
        qkv = (norm(x) @ f(w["qkv"])).reshape(n, H + 2 * G, D)
        t = norm(qkv[:, :H + G])
        a, b = t[..., :D // 2], t[..., D // 2:]
        t = np.concatenate((a * cos - b * sin, b * cos + a * sin), axis=-1)
        q, k, v = t[:, :H], held(t[:, H:]).repeat(H // G, axis=1), held(qkv[:, H + G:]).repeat(H // G, axis=1)
        s = np.einsum("ihd,jhd->hij", q, k) / math.sqrt(D)
        s = np.where(np.tri(n, dtype=bool), s, -np.inf)
        e = np.exp(s - s.max(-1, keepdims=True))
        x = x + np.einsum("hij,jhd->ihd", e / e.sum(-1, keepdims=True), v).reshape(n, -1) @ f(w["o"])
        y = norm(x)
        g = y @ f(w["gate"])
        x = x + (g / (1 + np.exp(-g)) * (y @ f(w["up"]))) @ f(w["down"])
    return norm(x) @ f(m.head)


@pytest.mark.parametrize("drafts,length,page", [(1, 4, 8), (3, 5, 16), (4, 8, 8)])
def test_caches_of_four_bits(example, drafts, length, page):  # noqa: F811
    """The text is the one that the target writes by itself over a cache of 4 bits.  The products in front of the cache are float32's, so an entry may lie on the other
    side of a border than in float64 and be a code off (a step of up to a third of itself, one entry in a few hundred thousand): a token is compared where the two
    likeliest logits are 0.05 apart."""
    import torch
    target, draft = _models(example, torch.float32)
    prompts = _prompts(500, (3, 8, 41))
    text, iterations, pool = example.decode_on_gpu(target, draft, prompts, drafts, length, new=24, page=page, top_k=1, top_p=1.0)
    assert 24 / (length + 1) <= iterations < 24
    _all_free(pool)
    compared = 0
    for p, t in zip(prompts, text):
        assert t[:len(p)] == p and len(t) >= len(p) + 24
        z = _held_logits(target, t)
        for i in range(len(p) - 1, len(t) - 1):
            best = np.sort(z[i])[-2:]
            if best[1] - best[0] >= 0.05:
                compared += 1
                assert t[i + 1] == int(z[i].argmax())
    assert compared >= 40


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("packed", [False, True])
def test_texts_of_one_seed_are_the_same(example, dtype, packed):  # noqa: F811
    import torch
    target, draft = _models(example, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype], V=700)
    prompts = _prompts(700, (1, 16, 30, 65))
    runs = [example.decode_on_gpu(target, draft, prompts, 4, 6, new=20, page=16, top_k=20, top_p=0.95, min_p=0.01, packed=packed) for _ in range(2)]
    assert runs[0][:2] == runs[1][:2]
    for pool in (runs[0][2], runs[1][2]):
        _all_free(pool)
    for p, t in zip(prompts, runs[0][0]):
        assert t[:len(p)] == p and len(p) + 20 <= len(t) <= len(p) + 26


@pytest.mark.parametrize("packed", [False, True])
def test_a_draft_model_that_is_the_target_is_always_right(example, packed):  # noqa: F811
    """Every drafted token is taken for as long as the draft model's pages hold what the text says, but where two tokens are nearly as likely."""
    import torch
    target, draft = _models(example, torch.float32, noise=0.0)
    prompts = _prompts(500, (3, 8, 17))
    for drafts, length, page in ((2, 4, 8), (1, 8, 8), (3, 7, 16)):
        text, iterations, _ = example.decode_on_gpu(target, draft, prompts, drafts, length, new=6 * (length + 1), page=page, top_k=1, top_p=1.0, packed=packed)
        near = 0
        for p, t in zip(prompts, text):
            best = np.sort((_held_logits if packed else _plain_logits)(target, t)[len(p) - 1:-1], axis=-1)[:, -2:]
            near += int((best[:, 1] - best[:, 0] < (0.05 if packed else 1e-3)).sum())
        assert 6 <= iterations <= 6 + near, (drafts, length, page, near)
