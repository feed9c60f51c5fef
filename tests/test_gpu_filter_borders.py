"""Borders of min_p and of the histogram's bins where float64's weights say little: entries whose weight rounds to that of the largest, and
borders next to 0, around which float32's values lie far closer together than the float64 differences to the largest logit (needs an MI355X: run
with -m gpu).  Kept sets and tokens are those of the definition in float64, but min_p = 1 keeps the entries that equal the largest, whatever
the others' weights round to."""
import numpy as np
import pytest

from decoding_util import plain_filter, torch_dtype

pytestmark = pytest.mark.gpu


def _check(z, dtype, label, **kw):
    import torch
    import paper_2604_25925_amd as sg
    x = torch.from_numpy(np.ascontiguousarray(z, np.float32)).cuda().to(torch_dtype(dtype))
    t = {n: torch.from_numpy(np.asarray(v, np.float32)).cuda() for n, v in kw.items()}
    u = t.pop("u")
    tokens, kept, _ = sg.specgbv_sample_filtered(x, u, keep=True, **t)
    torch.cuda.synchronize()
    xs, ks, tokens = x.float().cpu().numpy(), kept.float().cpu().numpy(), tokens.cpu().numpy()
    for r in range(len(xs)):
        f = {("T" if n == "temperature" else n): np.float32(v[r]) for n, v in kw.items()}
        z = xs[r]
        if f.get("min_p", 0) >= 1:
            z = np.where(z == z.max(), z, -np.inf)
        want, mask = plain_filter(z, **f)
        got = ks[r] > -np.inf
        assert np.array_equal(got, mask), "%s row %d: kept %d, want %d" % (label, r, got.sum(), mask.sum())
        assert tokens[r] == want, "%s row %d: token %d, want %d" % (label, r, tokens[r], want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,V", [(4, 50), (4, 3000), (300, 500)])
@pytest.mark.parametrize("scale,temperature", [(1e-25, 1.0), (1e-38, 0.5), (1e-17, 1.0), (1.0, 1e20), (30.0, 1e30), (1e-20, 1e-3)])
def test_weights_that_round_to_one(dtype, R, V, scale, temperature):
    rng = np.random.default_rng(V)
    z = rng.normal(0, 1, (R, V)).astype(np.float32) * np.float32(scale)
    for min_p in (1.0, 0.99999994, 0.5):
        _check(z, dtype, "%g %g %g" % (scale, temperature, min_p), temperature=[temperature] * R, min_p=[min_p] * R, u=rng.random(R).astype(np.float32))


def _border_next_to_zero():
    """(T, min_p) of float32 for which 1 + T ln(min_p) is nearly 0, on each side."""
    m = np.random.default_rng(1).uniform(0.05, 0.9, 4_000_000).astype(np.float32)
    T = (-1.0 / np.log(m.astype(np.float64))).astype(np.float32)
    at = 1.0 + T.astype(np.float64) * np.log(m.astype(np.float64))
    found = []
    for side in (at > 0, at < 0):
        i = np.argmin(np.where(side, np.abs(at), 1.0))
        assert 1e-15 < abs(at[i]) < 1e-12
        found.append((T[i], m[i], at[i]))
    return found


SMALL = [s * v for v in (0.0, 1e-45, 1e-40, 1e-30, 1e-20, 1e-18, 1e-15, 1e-12, 1e-9) for s in (1.0, -1.0)]


def test_a_min_p_whose_border_is_next_to_zero():
    rng = np.random.default_rng(2)
    for T, m, at in _border_next_to_zero():
        z = rng.normal(-3, 0.3, (6, 400)).astype(np.float32)
        for r in range(6):
            z[r, rng.choice(400, len(SMALL), replace=False)] = SMALL
            z[r, 5] = 1.0
        _check(z, "f32", "border at %g" % at, temperature=[T] * 6, min_p=[m] * 6, u=[0.0, 0.2, 0.5, 0.8, 0.95, 0.9999])


@pytest.mark.parametrize("bins", [0, 1, 3])
def test_a_bin_whose_border_is_next_to_zero(bins):
    """Bins are 1/64 of an octave of the weight, the nearest integers to 64 log2(e) (top - z) / T: a border next to z = 0, with many entries on
    both sides of it."""
    rng = np.random.default_rng(3)
    top = rng.uniform(0.5, 2.0, 4_000_000).astype(np.float32)
    per = 64.0 * 1.44269504088896340736
    T = (top.astype(np.float64) * per / (bins + 0.5)).astype(np.float32)
    at = top.astype(np.float64) - (bins + 0.5) * T.astype(np.float64) / per
    for side in (at > 0, at < 0):
        i = np.argmin(np.where(side & (np.abs(at) > 2e-15), np.abs(at), 1.0))
        assert abs(at[i]) < 1e-12
        z = rng.choice(np.float32(SMALL), (16, 400))
        z[:, 5] = top[i]
        _check(z, "f32", "border of a bin at %g" % at[i], temperature=[T[i]] * 16, top_p=[1.0] * 8 + list(np.linspace(0.3, 0.99, 8)), u=np.linspace(0.03, 0.97, 16))
