"""What the binding of the decoding step's operators makes of tensors, without a GPU: CPU tensors that say they live on one take the public
functions up to the C checks, which refuse the call before anything is launched."""
import pytest
import torch

import paper_2604_25925_amd as sg
import paper_2604_25925_amd.decoding  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses here are no GPU's: nothing may come to a launch")


class _Said(torch.Tensor):
    """A CPU tensor that says it lives on a GPU."""
    is_cuda = True


def _said(x):
    return x.as_subclass(_Said)


def _cache(S, width=4, pages=8, G=2, page=8, D=64, table=None, dtype=torch.bfloat16):
    k, v = (_said(torch.zeros((pages, G, page, D), dtype=dtype)) for _ in range(2))
    return sg.PagedCache(k, v, _said(torch.zeros((S, width), dtype=torch.int32) if table is None else table))


def _append(cache, positions, heads=4):
    S, T, D = cache.sequences, positions.shape[1], cache.head_dim
    q, k = (_said(torch.zeros((S, T, h, D), dtype=cache.dtype)) for h in (heads, cache.kv_heads))
    return sg.specgbv_cache_append(cache, q, k, k, positions, stream=0)


def _attend(cache, positions, heads=4, **kw):
    q = _said(torch.zeros((cache.sequences, positions.shape[1], heads, cache.head_dim), dtype=cache.dtype))
    return sg.specgbv_attend_paged(cache, q, positions, stream=0, **kw)


def _overlapping(S, n):
    """int32 [S, n] views whose rows lie closer together than they are long."""
    return [_said(torch.zeros((1, n), dtype=torch.int32).expand(S, n)), _said(torch.zeros(S + n - 1, dtype=torch.int32).unfold(0, n, 1))]


@pytest.mark.parametrize("call", [_append, _attend])
def test_rows_that_are_closer_than_they_are_long_are_refused(call):
    for positions in _overlapping(3, 5):
        assert positions.shape == (3, 5) and positions.stride(0) < 5
        with pytest.raises(sg.SpecGBVError) as e:
            call(_cache(3), positions)
        assert e.value.status == 1 and "positions_stride" in str(e.value)
    for table in _overlapping(3, 4):
        with pytest.raises(sg.SpecGBVError) as e:
            call(_cache(3, table=table), _said(torch.zeros((3, 2), dtype=torch.int32)))
        assert e.value.status == 1 and "table_stride" in str(e.value)


@pytest.mark.parametrize("stride", [0, 1, 7, 50])
def test_the_stride_of_a_single_row_is_of_no_matter(stride):
    one = _said(torch.zeros(60, dtype=torch.int32).as_strided((1, 5), (stride, 1)))
    assert _cache(1)._positions(one, 5) >= 5
    assert _cache(1, table=one).sequences == 1
    rows = _said(torch.zeros(60, dtype=torch.int32).as_strided((3, 5), (11, 1)))
    assert _cache(3)._positions(rows, 5) == 11


def _filtered(**kw):
    z = _said(torch.zeros((3, 40)))
    return sg.specgbv_sample_filtered(z, _said(torch.zeros(3)), stream=0, **kw)


def _verification(name, **kw):
    B, K, L, V = 1, 2, 3, 64
    target, draft, tokens = _said(torch.zeros((B, K, L + 1, V))), _said(torch.zeros((B, K, L, V))), _said(torch.zeros((B, K, L), dtype=torch.int32))
    one, nu = _said(torch.zeros(B, dtype=torch.int32)), _said(torch.zeros(B, dtype=torch.float64))
    if name in ("specgbv_verify", "specgbv_verify_ex", "specgbv_verify_kseq"):
        return getattr(sg, name)(target, draft, tokens, 1.0, 0, 0, stream=0, **kw)
    if name == "specgbv_modify_target":
        return sg.specgbv_modify_target(target, draft, tokens, 1.0, nu, one, stream=0, **kw)
    if name == "specgbv_sample_tokens":
        return sg.specgbv_sample_tokens(target, 1.0, 0, 0, 0, stream=0, **kw)
    return sg.specgbv_carry_advance(target, draft, tokens, one, one, _said(torch.zeros((B, L + 1), dtype=torch.int32)), 1.0, nu, one, stream=0, **kw)


@pytest.mark.parametrize("call", [lambda **kw: _attend(_cache(3), _said(torch.zeros((3, 2), dtype=torch.int32)), **kw), _filtered] +
                         [lambda name=name, **kw: _verification(name, **kw) for name in
                          ("specgbv_verify", "specgbv_verify_ex", "specgbv_verify_kseq", "specgbv_modify_target", "specgbv_sample_tokens", "specgbv_carry_advance")])
def test_a_workspace_is_dense_and_lives_on_the_calls_gpu(call):
    n = 1 << 24
    for workspace in (torch.zeros(n, dtype=torch.uint8),                                      # on the host
                      _said(torch.zeros(1, dtype=torch.uint8).expand(n)),                     # less memory than entries
                      _said(torch.zeros(4 * n, dtype=torch.uint8))[::4],
                      _said(torch.zeros(n, dtype=torch.uint8, device="meta"))):               # on another device
        with pytest.raises(ValueError, match="workspace"):
            call(workspace=workspace)


@pytest.mark.parametrize("shape", [(0, 40), (2, 0, 40), (0, 2, 40), (3, 0, 2, 40), (1, 0, 40)])
def test_logits_without_rows(shape):
    for z in (torch.zeros(shape), torch.zeros([n + 3 for n in shape[:-1]] + [50])[tuple(slice(0, n) for n in shape)]):
        assert z.shape == shape
        tokens, kept, _ = sg.specgbv_sample_filtered(_said(z), _said(torch.zeros(0)), keep=True, stream=0)
        assert tokens.shape == (0,) and kept.shape == shape


def test_caches_without_sequences_and_calls_without_tokens():
    for S, T in ((0, 1), (0, 0), (3, 0)):
        positions = _said(torch.zeros((S, T), dtype=torch.int32))
        assert _append(_cache(S), positions).shape == (S, T, 4, 64)
        assert _attend(_cache(S), positions)[0].shape == (S, T, 4, 64)
        assert _attend(_cache(S), positions, shared_len=_said(torch.zeros(S, dtype=torch.int32)))[0].shape == (S, T, 4, 64)


HINTS = [0, 1, 40, 200, 256, 257, 513, 900, 1024, 1025, 2048, 4000, 5000, 1 << 20]


@pytest.mark.parametrize("prefixes,drafts", [(1, 1), (1, 3), (3, 1), (4, 8), (32, 8), (70, 1), (70, 2), (300, 1)])
@pytest.mark.parametrize("window", [0, 700])
def test_a_workspace_serves_every_max_len(prefixes, drafts, window):
    """A loop that keeps its workspace while its text, and with it max_len, grows or starts anew."""
    for G, D, T, heads, dtype in ((8, 128, 8, 32, torch.bfloat16), (8, 128, 1, 32, torch.bfloat16), (1, 64, 1, 5, torch.float32), (2, 256, 9, 8, torch.bfloat16)):
        S = prefixes * drafts
        for shared in ([None, _said(torch.zeros(prefixes, dtype=torch.int32))] if drafts > 1 else [None]):
            cache = _cache(S, width=600, pages=1, G=G, D=D, dtype=dtype)
            q = _said(torch.zeros((1, 1, 1, 1), dtype=dtype).expand(S, T, heads, D).contiguous())
            need = {n: sg.specgbv_attend_workspace_bytes(cache, q, window=window, shared_len=shared, max_len=n) for n in HINTS}
            assert len(set(need.values())) == 1, (G, D, T, shared is None, need)
            positions = _said(torch.zeros((S, T), dtype=torch.int32))
            _, kept = _tried(cache, q, positions, window=window, shared_len=shared, max_len=200)      # what the binding makes for a short text
            for n in HINTS:
                status, _ = _tried(cache, q, positions, window=window, shared_len=shared, max_len=n, workspace=kept)
                assert status == 4, (G, D, T, shared is None, n)                                      # (no GPU: it came to the launch)


def _tried(cache, q, positions, workspace=None, **kw):
    """(status, workspace) of a call that comes as far as its launch."""
    made = []
    empty = torch.empty

    def keep(n, **kwargs):                                    # on a border of 256 bytes, as on a GPU
        room = empty(n + 256, **kwargs)
        at = -room.data_ptr() % 256
        made.append(_said(room[at:at + n]))
        return made[-1]
    torch.empty = keep
    try:
        sg.specgbv_attend_paged(cache, q, positions, stream=0, out=q, workspace=workspace, **kw)
    except sg.SpecGBVError as e:
        return e.status, workspace if workspace is not None else made[0]
    finally:
        torch.empty = empty


def _sizes(S, T, H, G, D=64, page=16, width=600, prefixes=0):
    """(cache, append's arguments, attention's arguments) of sizes that no tensors here have."""
    P = 1 << 20
    cache = sg.decoding._CACHE.pack(P, P, P, page * G * D, page * D, D, page * G * D, page * D, D, width, 9, G, page, D, S, width, 1, 0)
    q, kv = (T * H * D, H * D, D), (T * G * D, G * D, D)
    append = sg.decoding._APPEND.pack(P, P, P, P, P, 0, 0, 0, *q, *kv, *kv, *q, T, 1e-6, T, H, 0, 0)
    attend = sg.decoding._ATTEND.pack(P, P, P, P if prefixes else 0, *q, *q, T, T, H, 0, prefixes, 0, 0.0)
    return cache, append, attend


@pytest.mark.parametrize("S,T,H,G,fits", [(1, 2 ** 25 - 2, 8, 2, True), (1, 2 ** 25 - 1, 8, 2, False), (5 * 10 ** 7, 1, 4, 1, False), (2 ** 24, 2, 1, 1, False),
                                          (1, 1, 2 ** 29 - 2, 1, True), (1, 1, 2 ** 29, 1, False), (1, 1, 10 ** 9, 10 ** 9, False)])
def test_appends_that_no_launch_holds(S, T, H, G, fits):
    cache, append, _ = _sizes(S, T, H, G, D=8)
    assert sg.load_library().specgbv_cache_append(cache, append, None) == (4 if fits else 2), sg.specgbv_last_error()


@pytest.mark.parametrize("S,T,H,G,prefixes,fits", [(2 ** 21 - 1, 1, 8, 8, 0, True), (2 ** 21, 1, 8, 8, 0, False), (2, 2 ** 20 - 1, 128, 128, 1, True),
                                                   (2, 2 ** 20, 128, 128, 1, False)])
def test_attention_that_no_launch_holds(S, T, H, G, prefixes, fits):
    """By its own grid, and by that of the join behind it, before either is launched."""
    cache, _, attend = _sizes(S, T, H, G, prefixes=prefixes)
    assert sg.load_library().specgbv_attend_paged(cache, attend, 1 << 20, 1 << 50, None) == (4 if fits else 2), sg.specgbv_last_error()
