"""specgbv_sample_filtered against the definition in float64 (needs an MI355X: run with -m gpu).  Kept sets and tokens have to be equal:
the weights decide by float64 and by sums of integers of 2^-43 of the largest weight, and the inputs are drawn without regard to
borders, which lie within that of a goal once in 10^8 rows."""
import numpy as np
import pytest

from decoding_util import plain_filter, torch_dtype

pytestmark = pytest.mark.gpu


def _gpu(z, dtype, **kw):
    import torch
    import paper_2604_25925_amd as sg
    x = torch.from_numpy(np.ascontiguousarray(z, np.float32)).cuda().to(torch_dtype(dtype))
    t = {n: (None if v is None else torch.tensor(v, dtype=torch.int32 if n == "top_k" else torch.float32, device="cuda")) for n, v in kw.items()}
    u = t.pop("u", None)
    tok, kept, _ = sg.specgbv_sample_filtered(x, u, draw=u is not None, keep=True, **t)
    torch.cuda.synchronize()
    return x, (None if tok is None else tok.cpu().numpy()), kept


def _check(z, dtype, label="", **kw):
    x, tok, kept = _gpu(z, dtype, **kw)
    xs, ks = x.float().cpu().numpy(), kept.float().cpu().numpy()
    for r in range(xs.shape[0]):
        one = {("T" if n == "temperature" else n): (None if v is None else np.float32(v[r]) if n != "top_k" else int(v[r])) for n, v in kw.items()}
        want, mask = plain_filter(xs[r], **one)
        got = ks[r] > -np.inf
        assert np.array_equal(got, mask), "%s row %d: kept %d, want %d" % (label, r, got.sum(), mask.sum())
        assert np.array_equal(ks[r][mask], xs[r][mask])
        if tok is not None:
            assert tok[r] == want, "%s row %d: token %d, want %d" % (label, r, tok[r], want)


def _rows(rng, R, V, head=0, masked=0):
    z = rng.normal(0, 3, (R, V)).astype(np.float32)
    for r in range(R):
        if head:
            at = rng.choice(V, min(head, V), replace=False)
            z[r, at] += 6 - 1.1 * np.log(np.arange(1, len(at) + 1))
        if masked:
            z[r, V - masked:] = -np.inf
    return z


def _some(rng, R, kind):
    pick = lambda *v: rng.choice(v, R)
    f = dict(temperature=pick(0.4, 0.7, 1.0, 1.3), u=rng.random(R).astype(np.float32))
    if kind in ("top_k", "all"):
        f["top_k"] = pick(1, 2, 20, 50, 1000, 0)
    if kind in ("top_p", "all"):
        f["top_p"] = pick(0.1, 0.5, 0.9, 0.99, 1.0)
    if kind in ("min_p", "all"):
        f["min_p"] = pick(0.0, 0.01, 0.1, 0.9)
    return f


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["none", "top_k", "top_p", "min_p", "all"])
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (5, 7), (9, 64), (6, 515), (4, 4097), (3, 32003), (2, 70001), (2, 152064)])
def test_filters(dtype, kind, R, V):
    rng = np.random.default_rng(V * 7 + len(kind))
    _check(_rows(rng, R, V, head=50 if V > 100 else 0, masked=V // 100), dtype, "%s %d %s" % (kind, V, dtype), **_some(rng, R, kind))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,shift", [(0.0, 0.0), (1e-3, 0.0), (1.0, 200.0), (30.0, -500.0), (1e4, 0.0), (1e-30, 0.0)])
def test_scales_of_logits(dtype, scale, shift):
    """Rows of one value, of values close together (bins of thousands of entries) and far apart, around zero and far from it."""
    rng = np.random.default_rng(11)
    for V in (300, 5000, 40000):
        z = rng.normal(0, 1, (4, V)).astype(np.float32) * scale + shift
        for kind in ("none", "all"):
            _check(z, dtype, "scale %g shift %g %d" % (scale, shift, V), **_some(rng, 4, kind))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties(dtype):
    """Few values, each many times, both zeros among them: a cut within thousands of ties goes by the index."""
    rng = np.random.default_rng(5)
    for V in (40, 3000, 66000, 150001):
        z = rng.choice(np.array([-2.0, -0.0, 0.0, 0.5, 1.0], np.float32), (5, V), p=[0.1, 0.2, 0.2, 0.3, 0.2])
        z[1] = 1.25
        z[2, :] = np.where(np.arange(V) % 2, 0.0, -0.0)
        z[3, :-1] = -5.0
        for u in (0.0, 0.3, 0.77, 0.9999):
            _check(z, dtype, "ties %d" % V, temperature=[1.0, 0.5, 2.0, 1.0, 0.1], u=[u] * 5)
            _check(z, dtype, "ties %d" % V, top_k=[7, V // 3, V // 2, V, 1], u=[u] * 5)
            _check(z, dtype, "ties %d" % V, top_p=[0.37, 0.613, 0.499, 0.9, 0.2], u=[u] * 5)


def test_rows_beyond_16_bit_counts():
    """More than 65535 entries of one value, more than 2 x 65536 of two, and the longest row."""
    rng = np.random.default_rng(6)
    z = np.full((4, 150000), 0.5, np.float32)
    z[0, ::2] = 0.25
    z[1, 70000:] = rng.normal(0, 1, 80000)
    z[2, 1::3] = -np.inf
    z[3] = np.repeat(np.float32([1, 2]), 75000)
    f = dict(temperature=[1.0, 0.7, 1.0, 1.5], u=[0.1, 0.55, 0.9, 0.7])
    _check(z, "bf16", "many", **f)
    _check(z, "bf16", "many", top_p=[0.6, 0.9, 0.5, 0.95], top_k=[0, 100000, 99999, 80000], **f)
    z = rng.normal(0, 2, (2, 1 << 20)).astype(np.float32)
    z[1] = 3.0
    for dtype in ("bf16", "f32"):
        _check(z, dtype, "longest", temperature=[0.8, 1.0], top_p=[0.9, 0.7], u=[0.4, 0.8])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_entries_and_numbers_that_are_none(dtype):
    rng = np.random.default_rng(8)
    V = 3000
    z = rng.normal(0, 3, (9, V)).astype(np.float32)
    z[0] = -np.inf                                           # nothing to draw
    z[1, :] = -np.inf
    z[1, 1234] = -80.0                                       # one entry
    z[2, ::2] = -np.inf
    z[3, 5] = np.inf
    z[4, [7, 70, 700]] = np.inf
    z[5, ::3] = np.nan                                       # no number: as -inf
    z[6] = np.nan
    z[7] = np.finfo(np.float32).min if dtype == "f32" else -3.0e38
    z[8, :2990] = -3.0e38
    for f in (dict(), dict(top_k=[5] * 9), dict(top_p=[0.7] * 9), dict(min_p=[0.2] * 9)):
        for u in (0.0, 0.6, 0.999):
            _check(z, dtype, "masked", u=[u] * 9, **f)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_edges_of_parameters(dtype):
    rng = np.random.default_rng(9)
    z = _rows(rng, 8, 2000, head=20)
    u = rng.random(8).astype(np.float32)
    _check(z, dtype, "T", temperature=[0.0, -1.0, 1e-6, 1e-30, 1e6, 1e30, np.nan, 0.5], u=u)
    _check(z, dtype, "k", top_k=[-5, 0, 1, 1999, 2000, 2001, 2 ** 31 - 1, -2 ** 31], u=u)
    _check(z, dtype, "p", top_p=[-1.0, 0.0, 1e-30, 1.0, 2.0, 0.99999994, np.nan, 0.5], u=u)
    _check(z, dtype, "m", min_p=[-1.0, 0.0, 1e-30, 1.0, 5.0, 0.5, 1e-4, 0.99], u=u)
    _check(z, dtype, "u", temperature=[1.0] * 8, u=[0.0, 1e-30, 0.5, 0.99999994, 0.9, 0.1, 0.3, 0.7])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_in_place_and_odd_addresses(dtype):
    import torch
    import paper_2604_25925_amd as sg
    rng = np.random.default_rng(12)
    R, V = 6, 1003
    z = torch.from_numpy(rng.normal(0, 3, (R, 2, V + 5)).astype(np.float32)).cuda().to(torch_dtype(dtype))
    u = torch.from_numpy(rng.random(R).astype(np.float32)).cuda()
    p = torch.full((R,), 0.8, device="cuda")
    for shift in (0, 1, 3):
        view = z[:, 1, shift:shift + V]                      # the last position of each sequence, say
        ref_t, ref_k, _ = sg.specgbv_sample_filtered(view.contiguous(), u, top_p=p, keep=True)
        tok, kept, _ = sg.specgbv_sample_filtered(view, u, top_p=p, keep=True)
        assert torch.equal(tok, ref_t) and torch.equal(kept, ref_k)
        copy = z.clone()
        mine = copy[:, 1, shift:shift + V]
        tok, kept, _ = sg.specgbv_sample_filtered(mine, u, top_p=p, keep=True, kept=mine)
        assert torch.equal(tok, ref_t) and torch.equal(mine, ref_k)
        copy[:, 1, shift:shift + V] = z[:, 1, shift:shift + V]
        assert torch.equal(copy, z)                          # nothing beside the rows is written
        into = torch.zeros((R, V + 3), dtype=z.dtype, device="cuda")
        sg.specgbv_sample_filtered(view, top_p=p, draw=False, keep=True, kept=into[:, 2:2 + V])
        assert torch.equal(into[:, 2:2 + V], ref_k) and bool((into[:, :2] == 0).all()) and bool((into[:, V + 2:] == 0).all())
        three = view.unsqueeze(1)
        tok, _, _ = sg.specgbv_sample_filtered(three, u, top_p=p)
        assert torch.equal(tok, ref_t)


def test_tokens_follow_the_truncated_law():
    import scipy.stats
    rng = np.random.default_rng(4)
    n, V = 40000, 12
    row = rng.normal(0, 1.5, V).astype(np.float32)
    z = np.tile(row, (n, 1))
    _, tok, kept = _gpu(z, "f32", temperature=[0.9] * n, top_p=[0.85] * n, u=rng.random(n).astype(np.float32))
    _, mask = plain_filter(row, T=np.float32(0.9), top_p=np.float32(0.85))
    w = np.where(mask, np.exp(row.astype(np.float64) / np.float64(np.float32(0.9))), 0)
    counts = np.bincount(tok, minlength=V)
    assert counts[~mask].sum() == 0 and 1 < mask.sum() < V
    assert scipy.stats.chisquare(counts[mask], (w / w.sum())[mask] * n).pvalue > 1e-4


def test_refusals_and_empty_calls():
    import torch
    import paper_2604_25925_amd as sg
    z, u = torch.zeros((4, 64), device="cuda"), torch.zeros(4, device="cuda")
    for kw in (dict(u=u[:3]), dict(u=u.double()), dict(u=u, top_k=u), dict(u=u, top_p=u.cpu()), dict(u=None), dict(u=u, draw=False),
               dict(u=u, out=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(u=u, keep=True, kept=z[:, :32])):
        with pytest.raises(ValueError):
            sg.specgbv_sample_filtered(z, **kw)
    tok, _, _ = sg.specgbv_sample_filtered(z[:0], u[:0])
    assert tok.numel() == 0


def test_replays_of_a_captured_call():
    import torch
    import paper_2604_25925_amd as sg
    z = torch.empty((16, 5000), dtype=torch.bfloat16, device="cuda")
    u, p = torch.empty(16, device="cuda"), torch.full((16,), 0.9, device="cuda")
    k = torch.full((16,), 300, dtype=torch.int32, device="cuda")
    z.normal_()
    u.uniform_()
    tok, kept, ws = sg.specgbv_sample_filtered(z, u, top_p=p, top_k=k, keep=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sg.specgbv_sample_filtered(z, u, top_p=p, top_k=k, keep=True, out=tok, kept=kept, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sg.specgbv_sample_filtered(z, u, top_p=p, top_k=k, keep=True, out=tok, kept=kept, workspace=ws)
    for step in range(5):
        z.normal_(0, 1 + step)
        u.uniform_()
        t, kk, _ = sg.specgbv_sample_filtered(z, u, top_p=p, top_k=k, keep=True)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tok, t) and torch.equal(kept, kk)


@pytest.mark.parametrize("V", [300, 8191, 32000])
@pytest.mark.parametrize("kind", ["none", "top_p", "all"])
def test_more_rows_than_compute_units(V, kind):
    """Rows of a large batch, among them ones that hold very small and very large magnitudes, zeros of both signs, infinities,
    numbers that are none, one value alone, and nothing."""
    rng = np.random.default_rng(V)
    R = 270
    z = _rows(rng, R, V, head=50, masked=V // 100)
    z[::5, 3] = 0.0
    z[::5, 7] = -0.0
    z[1, ::2] *= 1e-30
    z[2, 5] = 2.0 ** -63
    z[3, :] = 2.0 ** 65 * (1 + rng.random(V))
    z[4, 9:20] = [2.0 ** 66, -2.0 ** 66, 2.0 ** 64, -2.0 ** 64, 1e38, -1e38, 2.0 ** -62, -2.0 ** -62, 2.0 ** -64, -2.0 ** -64, 1e-38]
    z[6, 11] = np.inf
    z[7, ::3] = np.nan
    z[8, :] = -np.inf
    z[9, :] = 0.0
    z[11, :] = -np.inf
    z[11, V // 2] = -3.0
    z[12, :] = -rng.random(V) - 1
    z[13, :] = -3.0e38
    z[14, 0], z[14, V - 1] = -np.inf, 40.0
    kw = _some(rng, R, kind)
    _check(z, "bf16", "%s %d" % (kind, V), **kw)


@pytest.mark.parametrize("V", [1001, 8190, 32003, 40001])
def test_many_odd_rows_in_place(V):
    """Rows whose first and last 16 bytes hold a neighbour's entries, which the neighbour's workgroup overwrites meanwhile."""
    import torch
    import paper_2604_25925_amd as sg
    R = min(3000, 40_000_000 // V)
    gen = torch.Generator(device="cuda").manual_seed(V)
    z = (torch.randn((R, V), generator=gen, device="cuda") * 3).bfloat16()
    u = torch.rand(R, generator=gen, device="cuda")
    kw = dict(top_p=torch.full((R,), 0.9, device="cuda"), top_k=torch.full((R,), 300, dtype=torch.int32, device="cuda"))
    tokens, kept, _ = sg.specgbv_sample_filtered(z, u, keep=True, **kw)
    for _ in range(3):
        x = z.clone()
        mine, _, _ = sg.specgbv_sample_filtered(x, u, keep=True, kept=x, **kw)
        assert torch.equal(mine, tokens) and torch.equal(x, kept)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_min_p_that_is_no_number_is_off(dtype):
    rng = np.random.default_rng(4)
    _check(_rows(rng, 3, 2000, head=20), dtype, "nan", min_p=[np.nan, 0.05, -np.inf], u=rng.random(3).astype(np.float32))


@pytest.mark.parametrize("dtype,R,V", [("bf16", 530, 33001), ("bf16", 300, 100003), ("f32", 300, 9001)])
def test_batches_of_longer_rows(dtype, R, V):
    """More rows than compute units, of lengths that other forms of the kernel take: the next row loaded ahead, rows at odd addresses."""
    rng = np.random.default_rng(V)
    z = _rows(rng, R, V, head=50, masked=V // 100)
    z[3, :] = -np.inf
    z[R - 1, ::2] = np.nan
    _check(z, dtype, "%d" % V, **_some(rng, R, "all"))
