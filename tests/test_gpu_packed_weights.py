"""Float32 attention over a cache held in 4 bits: queries and weights with all their 24 bits; and powers of two of every byte."""
import numpy as np
import pytest

import paper_2604_25925_amd as sg
from decoding_util import host, torch_dtype
from packed_util import CODES
from packed_weights_util import LIVE, ONE, WAYS, bound, put_codes, queries, weights, zero_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [32, 8])
@pytest.mark.parametrize("way", list(WAYS))
@pytest.mark.parametrize("D,T", [(64, 1), (64, 5), (96, 3), (128, 1), (128, 17), (256, 1), (256, 5)])
def test_float32_queries_and_weights_have_all_their_bits(D, T, way, page):
    import torch
    gen = np.random.default_rng(D + T)
    S, G, length = WAYS[way]
    H, width = 2 * G, (length + page - 1) // page
    cache = zero_cache(gen, S, width, page, G, D, "f32")
    where = np.stack([np.sort(gen.permutation(length - T)[:LIVE]) for _ in range(S)])
    every = np.tile(np.arange(length), (S, 1))
    keys, values = np.zeros((S, length, G, D), np.uint8), gen.integers(0, 16, (S, length, G, D)).astype(np.uint8)
    keys[..., 0] = ONE                                       # weight 0
    values[..., :LIVE] = gen.integers(0, 16, (S, length, G, LIVE))
    for s in range(S):
        keys[s, where[s]] = 0
        values[s, where[s]] = 0
        for i, n in enumerate(where[s]):
            keys[s, n, :, 1 + i] = ONE
            values[s, n, :, i] = ONE
    put_codes(cache, "k", every, keys)
    put_codes(cache, "v", every, values)
    q = queries(gen, (S, T, H, D))
    positions = torch.tensor([[length - T + t for t in range(T)]] * S, dtype=torch.int32, device="cuda")
    print("case", D, T, way, page, flush=True)
    got = host(sg.specgbv_packed_attend(cache, torch.from_numpy(q).cuda(), positions, scale=1.0)[0])
    want = weights(q)
    off = np.abs(got[..., :LIVE] / want - 1)
    assert off.max() <= bound(), "%.3g times the bound at %s" % (off.max() / bound(), np.unravel_index(off.argmax(), off.shape))
    assert not got[..., LIVE:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_power_and_code_is_read_as_it_is(dtype):
    """Powers from 2^-127 to 2^125, as bytes 0 to 252 of a cache that a program laid out itself: tokens read back, and as the only token's value."""
    import torch
    gen = np.random.default_rng(30)
    S, G, D, page, width = 1, 2, 64, 16, 16                 # 256 tokens: one for each byte
    cache = zero_cache(gen, S, width, page, G, D, dtype)
    every = np.arange(256)[None]
    rows = np.tile(np.arange(D) % 16, (S, 256, G, 1)).astype(np.uint8)
    put_codes(cache, "k", every, rows)
    put_codes(cache, "v", every, rows)
    table = cache.table.cpu().numpy()
    for x in (cache.k_scale, cache.v_scale):
        byte = x.cpu().numpy()
        byte[table[0, every[0] // page], :, :, every[0] % page] = np.minimum(every[0], 252)[:, None, None]
        x.copy_(torch.from_numpy(byte))
    want = CODES[rows[0]] * 2.0 ** (np.minimum(every[0], 252) - 127.0)[:, None, None]
    k, v = sg.specgbv_packed_read(cache, torch.from_numpy(every.astype(np.int32)).cuda())
    for name, got in (("k", k), ("v", v)):
        wrong = np.flatnonzero((host(got)[0] != want).any((1, 2)))
        assert not wrong.size, (name, wrong[:8])
    q = torch.zeros((S, 256, G, D), dtype=torch_dtype(dtype), device="cuda")
    at = torch.from_numpy(every.astype(np.int32)).cuda()
    got = host(sg.specgbv_packed_attend(cache, q, at, window=1)[0])[0]
    wrong = np.flatnonzero((got != want).any((1, 2)))
    assert not wrong.size, ("attend", wrong[:8], got[wrong[:1]], want[wrong[:1]])
