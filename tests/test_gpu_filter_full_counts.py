"""Rows of bfloat16 whose 16-bit counts just hold, or just do not hold, all that is counted (needs an MI355X: run with -m gpu).  A row is counted
from the 16-byte border in front of it on, and what lies next to it counts as -inf, whose magnitude is that of +inf."""
import numpy as np
import pytest

from decoding_util import plain_filter

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [65520, 65527, 65528, 65529, 65530, 65535, 65536, 65543])
def test_rows_of_one_magnitude_at_every_address(V):
    import torch
    import paper_2604_25925_amd as sg
    rng = np.random.default_rng(V)
    for lead in range(8):
        z = np.full((4, V), np.inf, np.float32)
        z[1, ::2] = -np.inf                                  # the other sign's count
        z[2] = 1.5
        z[3, V // 2:] = -1.5
        z[3, :V // 2] = 1.5
        room = torch.full((4, V + 16 + 8 - (V + 16) % 8), 3.0, dtype=torch.bfloat16, device="cuda")      # rows a multiple of 16 bytes apart
        x = room[:, lead:lead + V]
        x.copy_(torch.from_numpy(z))
        u = rng.random(4).astype(np.float32)
        u[0] = 0.75
        tokens, kept, _ = sg.specgbv_sample_filtered(x, torch.from_numpy(u).cuda(), top_k=torch.tensor([0, 5, V - 1, V // 2 + 3], dtype=torch.int32, device="cuda"),
                                                     keep=True)
        torch.cuda.synchronize()
        got = kept.float().cpu().numpy() > -np.inf
        for r, k in enumerate((0, 5, V - 1, V // 2 + 3)):
            want, mask = plain_filter(z[r], top_k=k, u=u[r])
            assert int(tokens[r]) == want, (V, lead, r)
            assert np.array_equal(got[r], mask), (V, lead, r)
