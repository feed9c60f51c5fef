"""Attention over a cache held in 4 bits where references lie far from 0: known results, and rows that do not hang on the rows next to them."""
import numpy as np
import pytest

import paper_2604_25925_amd as sg
from decoding_util import host, torch_dtype
from packed_util import CODES, make_packed
from packed_weights_util import ONE, WAYS, put_codes, zero_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("way,page", [("one pass", 16), ("parts", 32), ("waves", 8), ("filled", 16)])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 256)])
def test_scores_far_beyond_what_a_product_is_exact_for(dtype, D, way, page):
    """A score is 64 * 2^p plus a small whole number, with c = scale log2(e) exactly 1, so that weights are powers of two and results known; and with c = 1.1, where a score
    times c has no exact float32 and equal scores must still weigh the same."""
    import torch
    gen = np.random.default_rng(D)
    S, G, length = WAYS[way]
    T, H, width = 2, 2 * G, (length + page - 1) // page
    cache = zero_cache(gen, S, width, page, G, D, dtype)
    every = np.tile(np.arange(length), (S, 1))
    keys, values = np.zeros((S, length, G, D), np.uint8), gen.integers(0, 16, (S, length, G, D)).astype(np.uint8)
    gaps = gen.choice([0, 1, 2, 3, 6], (S, length))          # below the largest score
    keys[..., 0] = ONE
    keys[..., D - 1] = np.select([gaps == g for g in (0, 1, 2, 3)], [0, 1 + 8, 2 + 8, 3 + 8], 5 + 8)[..., None]       # -0, -1/2, -1, -3/2, -3
    put_codes(cache, "k", every, keys)
    put_codes(cache, "v", every, values)
    v = CODES[values]
    positions = torch.tensor([[length - 2, length - 1]] * S, dtype=torch.int32, device="cuda")
    for large in (2.0 ** 15, 2.0 ** 21, 2.0 ** 23, -2.0 ** 21, -2.0 ** 23):
        x = np.zeros((S, T, H, D), np.float32)
        x[..., 0], x[..., D - 1] = large, 2.0
        q = torch.from_numpy(x).cuda().to(torch_dtype(dtype))
        print("case", dtype, D, way, page, large, flush=True)
        got = host(sg.specgbv_packed_attend(cache, q, positions, scale=float(np.float32(np.log(2.0))))[0])
        for t in range(T):
            w = 2.0 ** -gaps[:, :length - 1 + t].astype(np.float64)
            w /= w.sum(-1, keepdims=True)
            for g in range(G):
                want, mass = (np.einsum("sj,sjd->sd", w, z[:, :length - 1 + t, g]) for z in (v, np.abs(v)))
                # whole numbers below 2^24 and powers of two: the sums round, and the result
                err = mass * (length + 64) * 2.0 ** -23 + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 0.0)
                assert (np.abs(got[:, t, 2 * g:2 * g + 2] - want[:, None]) <= err[:, None]).all(), (large, t, g)
    # equal scores, whatever they are: the mean of the values
    keys[..., D - 1] = 0
    put_codes(cache, "k", every, keys)
    for large in (3.0, 12345.0, 2.0 ** 27 + 1000, 1e30, -2.0 ** 27 - 1000, -1e30):
        x = np.zeros((S, T, H, D), np.float32)
        x[..., 0] = large
        q = torch.from_numpy(x).cuda().to(torch_dtype(dtype))
        print("case equal", dtype, D, way, page, large, flush=True)
        got = host(sg.specgbv_packed_attend(cache, q, positions, scale=1.1 * float(np.log(2.0)))[0])
        for t in range(T):
            for g in range(G):
                want, mass = (z[:, :length - 1 + t, g].mean(1) for z in (v, np.abs(v)))
                # (the weights are all the same, but a power of two only where the reference is exact: bfloat16 rounds them)
                err = mass * ((length + 64) * 2.0 ** -23 + (2.0 ** -8 if dtype == "bf16" else 0.0)) * (1 + 2.0 ** -8) + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 0.0)
                assert (np.abs(got[:, t, 2 * g:2 * g + 2] - want[:, None]) <= err[:, None]).all(), (large, t, g)


@pytest.mark.parametrize("way,page", [("one pass", 16), ("parts", 32), ("waves", 8), ("filled", 16)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_rows_do_not_hang_on_vast_scores_next_to_them(D, way, page):
    """The queries of a kv head stand next to each other: the first ones' scores pass 2^20 or do not, and the others' results are the same bits."""
    import torch
    gen = np.random.default_rng(D + 1)
    S, G, length = WAYS[way]
    T, H, width = 1, 4 * G, (length + page - 1) // page
    cache = make_packed(gen, S, width, page, G, D, "f32")
    positions = torch.full((S, T), length - 1, dtype=torch.int32, device="cuda")
    q = torch.from_numpy(gen.normal(0, 1, (S, T, H, D)).astype(np.float32)).cuda()
    print("case", D, way, page, flush=True)
    alone = sg.specgbv_packed_attend(cache, q, positions, scale=0.3)[0]
    far = q.clone()
    far[:, :, ::4] *= 2.0 ** 24
    beside = sg.specgbv_packed_attend(cache, far, positions, scale=0.3)[0]
    assert torch.isfinite(beside).all()
    for h in (1, 2, 3):
        assert torch.equal(beside[:, :, h::4], alone[:, :, h::4]), (h, float((beside[:, :, h::4] - alone[:, :, h::4]).abs().max()))
