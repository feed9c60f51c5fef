"""specgbv_attend_paged over whole prompts and long chunks of them (needs an MI355X: run with -m gpu): queries drawn from all of them, the
first and the last among them, against the definition in float64, with decoding_util.attend_bound's bounds."""
import numpy as np
import pytest

from decoding_util import check_attend, make_cache, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,H,G,page,T,behind,window", [("bf16", 128, 8, 2, 16, 2050, 0, 0), ("bf16", 64, 4, 1, 64, 4001, 0, 0), ("f32", 64, 4, 4, 32, 1500, 0, 300),
                                                              ("bf16", 256, 2, 1, 16, 700, 0, 0), ("bf16", 128, 7, 1, 16, 512, 5000, 0), ("f32", 128, 3, 1, 8, 400, 1333, 0)])
def test_prompts(dtype, D, H, G, page, T, behind, window):
    import torch
    import paper_2604_25925_amd as sg
    S, width = 3, -(-(T + behind) // page)
    rng = np.random.default_rng(T + D)
    k, v, table = make_cache(rng, S, width, page, G, D, dtype, token_major=D == 64)
    q = torch.from_numpy(rng.normal(0, 1.5, (S, T, H, D)).astype(np.float32)).cuda().to(torch_dtype(dtype))
    length = np.array([T, T // 3, 1])                        # padded behind
    pos = np.where(np.arange(T) < length[:, None], behind + np.arange(T), -1).astype(np.int32)
    p = torch.from_numpy(pos).cuda()
    out, _ = sg.specgbv_attend_paged(sg.PagedCache(k, v, table), q, p, window=window)
    torch.cuda.synchronize()
    assert bool((out[p < 0] == 0).all())
    some = torch.from_numpy(np.unique(np.concatenate(([0, 1, T // 3 - 1, T // 3, T - 1], rng.integers(0, T, 9))))).cuda()
    check_attend(out[:, some], q[:, some], k, v, table, p[:, some], dtype, window)
