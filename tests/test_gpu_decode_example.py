"""The example of a decoding loop, which runs append, attention, truncated sampling and verification together (needs an MI355X: run with
-m gpu)."""
import importlib.util
import math
import pathlib

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = pathlib.Path(__file__).resolve().parents[1] / "examples" / "speculative_decode.py"
    spec = importlib.util.spec_from_file_location("speculative_decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _plain_logits(m, text):
    """Logits [tokens, V] of a text in float64 on the CPU, without a cache."""
    def f(w):
        return w.detach().double().cpu().numpy()

    def norm(x):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)

    n, D, H, G = len(text), m.D, m.heads, m.kv_heads
    x = f(m.embed)[np.asarray(text)]
    angle = np.arange(n)[:, None] * f(m.inv_freq)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    for w in m.layers:
        qkv = (norm(x) @ f(w["qkv"])).reshape(n, H + 2 * G, D)
        t = norm(qkv[:, :H + G])
        a, b = t[..., :D // 2], t[..., D // 2:]
        t = np.concatenate((a * cos - b * sin, b * cos + a * sin), axis=-1)
        q, k, v = t[:, :H], t[:, H:].repeat(H // G, axis=1), qkv[:, H + G:].repeat(H // G, axis=1)
        s = np.einsum("ihd,jhd->hij", q, k) / math.sqrt(D)
        s = np.where(np.tri(n, dtype=bool), s, -np.inf)
        e = np.exp(s - s.max(-1, keepdims=True))
        x = x + np.einsum("hij,jhd->ihd", e / e.sum(-1, keepdims=True), v).reshape(n, -1) @ f(w["o"])
        y = norm(x)
        g = y @ f(w["gate"])
        x = x + (g / (1 + np.exp(-g)) * (y @ f(w["up"]))) @ f(w["down"])
    return norm(x) @ f(m.head)


def _prompts(V, lengths):
    rng = np.random.default_rng(5)
    return [rng.integers(0, V, n).tolist() for n in lengths]


@pytest.mark.parametrize("drafts,length,page", [(1, 4, 8), (3, 5, 16), (4, 8, 8)])
def test_the_likeliest_tokens_are_those_of_the_target_alone(example, drafts, length, page):
    """top_k 1 leaves one token a row: whatever the drafts are, the text is the one that the target writes by itself.  A token is
    compared where the plain logits of the two likeliest ones are 1e-3 apart, far beyond float32's errors over two layers."""
    import torch
    target = example.Model(1, V=500, E=128, D=64, dtype=torch.float32)
    draft = example.Model(2, dtype=torch.float32, V=500, E=128, D=64, like=target, noise=0.7)
    prompts = _prompts(500, (3, 8, 41))
    text, iterations = example.decode(target, draft, prompts, drafts, length, new=24, page=page, top_k=1, top_p=1.0)
    assert 24 / (length + 1) <= iterations < 24               # drafted tokens were taken
    for p, t in zip(prompts, text):
        assert t[:len(p)] == p and len(t) >= len(p) + 24
        z = _plain_logits(target, t)
        for i in range(len(p) - 1, len(t) - 1):
            best = np.sort(z[i])[-2:]
            assert t[i + 1] == int(z[i].argmax()) or best[1] - best[0] < 1e-3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sampled_texts_stay_among_what_the_target_keeps(example, dtype):
    """Every new token is one that top_k 20 of the target keeps; a run with the same seed gives the same text."""
    import torch
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    target = example.Model(1, V=700, E=128, D=64, dtype=dt)
    draft = example.Model(2, dtype=dt, V=700, E=128, D=64, like=target, noise=0.7)
    prompts = _prompts(700, (1, 16, 30, 65))
    text, _ = example.decode(target, draft, prompts, 4, 6, new=20, page=16, top_k=20, top_p=0.95, min_p=0.01)
    again, _ = example.decode(target, draft, prompts, 4, 6, new=20, page=16, top_k=20, top_p=0.95, min_p=0.01)
    assert text == again
    if dtype == "f32":
        for p, t in zip(prompts, text):
            z = _plain_logits(target, t)
            for i in range(len(p) - 1, len(t) - 1):
                assert z[i, t[i + 1]] >= np.sort(z[i])[-20] - 1e-3
