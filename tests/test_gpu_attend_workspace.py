"""One workspace for a text that grows: calls of specgbv_attend_paged with different max_len (needs an MI355X: run with -m gpu)."""
import numpy as np
import pytest

from decoding_util import check_attend, make_cache, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,S,T,H,G,D,width", [("bf16", 1, 1, 8, 2, 128, 300), ("f32", 2, 3, 4, 1, 64, 260), ("bf16", 70, 1, 2, 1, 64, 70)])
def test_a_workspace_is_kept_while_sequences_grow(dtype, S, T, H, G, D, width):
    import torch
    import paper_2604_25925_amd as sg
    page = 16
    rng = np.random.default_rng(S + D)
    k, v, table = make_cache(rng, S, width, page, G, D, dtype)
    q = torch.from_numpy(rng.normal(0, 1.5, (S, T, H, D)).astype(np.float32)).cuda().to(torch_dtype(dtype))
    cache, ws = sg.PagedCache(k, v, table), None
    for max_len in (200, 257, 1025, width * page, 40):
        last = rng.integers(0, min(max_len, width * page), (S, 1))
        last[0] = min(max_len, width * page) - 1
        pos = torch.from_numpy(np.maximum(last - T + 1 + np.arange(T), -1).astype(np.int32)).cuda()
        out, ws = sg.specgbv_attend_paged(cache, q, pos, max_len=max_len, workspace=ws)
        torch.cuda.synchronize()
        check_attend(out, q, k, v, table, pos, dtype, label=str(max_len))
        ws.fill_(255)
