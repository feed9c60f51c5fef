"""Codes of turned keys at far positions, next to borders."""
import numpy as np
import pytest

import paper_2604_25925_amd as sg
from packed_exact_util import check_bytes, marked_cache, on_gpu, turned, turns
from packed_util import BORDERS

pytestmark = pytest.mark.gpu


def _next_to(border, cos, sin, gen, least, most):
    """A float32 pair (a, b) with a cos - b sin between `least` and `most` away from a border, on a side by chance; None where there is none."""
    b = np.round(gen.uniform(-1, 1, 1 << 17) * 2.0 ** 22) * 2.0 ** -22
    a = ((border + b * sin) / cos).astype(np.float32)
    rest = np.abs(a * cos - b * sin - border)
    fits = np.flatnonzero((rest > least) & (rest < most))
    return (float(a[fits[0]]), float(b[fits[0]])) if fits.size else None


@pytest.mark.parametrize("interleaved", [False, True])
def test_turned_entries_next_to_borders_at_far_positions(interleaved):
    """float32 pairs whose first entry lies 2^-45 to 2^-36 from a border once it is turned, at positions whose angle in float64 is 2^-36 to 2^-23 off: a block's power is set
    by an entry that does not turn, so the code shows on which side of the border the kernel saw it."""
    import torch
    gen = np.random.default_rng(20)
    D, R, page = 64, 8, 1 << 14
    positions = [131071, 131072 + 77, 1048575, 5000003, (1 << 26) + 12345, 987654321, (1 << 30) - 1]
    inv_freq = gen.uniform(0.5, 1.0, R)
    cos, sin = turns(positions, inv_freq)
    x = np.zeros((1, len(positions), 1, D), np.float32)
    x[..., 31] = 4.0
    found = 0
    for t in range(len(positions)):
        for r in range(R):
            if abs(cos[t, r]) < 0.8:                         # (so that no entry passes 7, which would be another power)
                continue
            pair = _next_to(float(gen.choice(BORDERS[2:6])), cos[t, r], sin[t, r], gen, 2.0 ** -45, 2.0 ** -36)
            if pair is not None:
                a, b = (2 * r, 2 * r + 1) if interleaved else (r, r + R)
                x[0, t, 0, a], x[0, t, 0, b] = pair
                found += 1
    assert found >= 12
    width = (1 << 30) // page
    table = np.full((1, width), -1, np.int32)
    for i, n in enumerate(sorted({p // page for p in positions})):
        table[0, n] = i
    cache, before = marked_cache(torch.from_numpy(table).cuda(), int(table.max()) + 1, page, 1, D, "f32")
    k = on_gpu(x)
    pos = np.array([positions])
    print("far turns", interleaved, found, flush=True)
    sg.specgbv_packed_append(cache, k, k, k, torch.tensor(pos, dtype=torch.int32, device="cuda"), inv_freq=torch.from_numpy(inv_freq).cuda(), interleaved=interleaved)
    y, off = turned(k, pos, inv_freq, interleaved=interleaved)
    left = check_bytes(cache, "k", before["k"], y, off, pos)
    assert left == 0                                          # (nothing is as near as the kernel's own error)
