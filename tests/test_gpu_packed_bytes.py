"""Every byte of a packed cache after an append, entry by entry: what is next to a border may have one of two codes, all else is as the definition says, and what no
token has is as it was."""
import numpy as np
import pytest

import paper_2604_25925_amd as sg
from decoding_util import host
from packed_exact_util import check_bytes, marked_cache, on_gpu, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 224, 256])
def test_every_byte_after_an_append(D, dtype):
    """Norms, rotations of all and of some entries, positions 0, near and far, padding: every code and power of every token, and every byte that is no token's."""
    import torch
    gen = np.random.default_rng(D + 300)
    S, T, H, G, page, width = 2, 4, 4, 2, 16, 9
    pos = np.array([[0, 1, 2, 143], [70, -1, 33, 144]])
    for norm in (False, True):
        for pairs in (0, D // 2, D // 4, 3):
            for interleaved in (False, True):
                label = (D, dtype, norm, pairs, interleaved)
                print("case", label, flush=True)
                table = torch.from_numpy(gen.permutation(S * width + 2)[:S * width].astype(np.int32).reshape(S, width)).cuda()
                cache, before = marked_cache(table, S * width + 2, page, G, D, dtype)
                q, k, v = (on_gpu(gen.normal(0, 1, (S, T, n, D)), dtype) for n in (H, G, G))
                inv_freq = 10000.0 ** (-np.arange(pairs) / max(pairs, 1))
                weight = on_gpu(1 + 0.3 * gen.normal(0, 1, D), dtype) if norm else None
                sg.specgbv_packed_append(cache, q, k, v, torch.tensor(pos, dtype=torch.int32, device="cuda"), interleaved=interleaved, k_weight=weight, eps=1e-5,
                                         inv_freq=torch.from_numpy(inv_freq).cuda() if pairs else None)
                y, off = turned(k, pos, inv_freq, weight, 1e-5, interleaved)
                left = check_bytes(cache, "k", before["k"], y, off, pos, label)
                assert left <= 2, label
                assert check_bytes(cache, "v", before["v"], host(v).astype(np.longdouble), np.zeros(v.shape, np.longdouble), pos, label) == 0
