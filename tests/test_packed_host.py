"""CPU-only checks of the operators on a cache held in 4 bits, of block tables and of slot maps: the layout of their C structures, every
refusal that the host makes before a launch, and what the binding looks at."""
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2604_25925_amd as sg
from paper_2604_25925_amd import decoding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                                  # an address that is never looked at: every call is refused before

FIELDS = {
    "specgbv_packed_cache": (decoding._PACKED, "k v k_scale v_scale table k_page_stride k_head_stride k_token_stride v_page_stride v_head_stride v_token_stride "
                             "k_scale_page_stride k_scale_head_stride k_scale_block_stride v_scale_page_stride v_scale_head_stride v_scale_block_stride table_stride "
                             "pages kv_heads page_size head_dim sequences table_width dtype reserved"),
    "specgbv_read_args": (decoding._READ, "k v positions k_stride v_stride positions_stride tokens reserved"),
    "specgbv_page_pool": (decoding._POOL, "table ring ends held table_stride pages page_size prefixes drafts table_width reserved"),
    "specgbv_advance_args": (decoding._ADVANCE, "length chosen shared_len served room reserved"),
    "specgbv_slot_args": (decoding._SLOTS, "table start count positions slots table_stride positions_stride slots_stride sequences drafts table_width page_size pages "
                          "tokens right reserved"),
}


def test_packed_arguments_have_the_c_structures_layout(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "%s"' % os.path.join(ROOT, "include", "specgbv.h"), 'int main(void) {']
    for name, (_, fields) in FIELDS.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        for f in fields.split():
            lines.append('printf("%s.%s %%zu %%zu\\n", offsetof(%s, %s), sizeof(((%s *)0)->%s));' % (name, f, name, f, name, f))
    (tmp_path / "layout.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run([cc, "-std=c99", "-o", str(tmp_path / "layout"), str(tmp_path / "layout.c")], check=True)
    got = dict(l.split(" ", 1) for l in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines())
    header = open(os.path.join(ROOT, "include", "specgbv.h")).read()
    for name, (packer, fields) in FIELDS.items():
        assert int(got[name]) == packer.size, name
        body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct \{([^}]*)\} %s;" % name, header).group(1), flags=re.S)
        declared = [re.sub(r"\[\d+\]|\W", "", x) for d in body.split(";") if d.strip() for x in re.sub(r"^\s*(const\s+)?\w+", "", d.strip()).split(",")]
        assert declared == fields.split(), name
        at = 0                                               # no gaps: the packed order is the declared one
        for f in fields.split():
            offset, size = map(int, got["%s.%s" % (name, f)].split())
            assert offset == at, (name, f)
            at += size
        assert at == packer.size


def _cache(**kw):
    a = dict(k=P, v=P, ks=P, vs=P, table=P, kp=2048, kh=512, kt=32, vp=2048, vh=512, vt=32, ksp=128, ksh=32, ksb=16, vsp=128, vsh=32, vsb=16, ts=5, pages=9, G=4, page=16,
             D=64, S=3, width=5, dtype=1)
    a.update(kw)
    return decoding._PACKED.pack(*[a[x] or 0 for x in "k v ks vs table kp kh kt vp vh vt ksp ksh ksb vsp vsh vsb ts pages G page D S width dtype".split()], 0)


BAD_CACHES = [(dict(dtype=2), 1), (dict(pages=0), 1), (dict(G=0), 1), (dict(S=-1), 1), (dict(width=0), 1), (dict(page=0), 1), (dict(D=0), 1), (dict(D=40), 2), (dict(D=288), 2),
              (dict(page=12), 2), (dict(width=1 << 20, ts=1 << 20, page=1 << 11), 2), (dict(ts=4), 1), (dict(kt=-32), 1), (dict(kt=40), 2), (dict(vh=1 << 31), 2), (dict(vp=24), 2),
              (dict(kt=(1 << 26) + 16), 2), (dict(ksb=-8), 1), (dict(ksb=12), 2), (dict(vsp=1 << 31), 2), (dict(vsb=(1 << 26) + 8), 2), (dict(k=None), 1), (dict(v=None), 1),
              (dict(ks=None), 1), (dict(vs=None), 1), (dict(table=None), 1), (dict(k=P + 8), 2), (dict(v=P + 8), 2), (dict(ks=P + 4), 2), (dict(vs=P + 4), 2), (dict(table=P + 2), 1)]


def _append(cache=None, args=True, **kw):
    a = dict(q=P, k=P, v=P, out=P, pos=P, freq=P, qw=0, kw=0, qs=(512, 512, 64), ks=(256, 256, 64), vs=(256, 256, 64), os=(512, 512, 64), ps=1, eps=1e-6, T=1, H=8, pairs=32,
             inter=0)
    a.update(kw)
    packed = decoding._APPEND.pack(*[a[x] or 0 for x in "q k v out pos freq qw kw".split()], *a["qs"], *a["ks"], *a["vs"], *a["os"], a["ps"], a["eps"], a["T"], a["H"], a["pairs"],
                                   a["inter"])
    return sg.load_library().specgbv_packed_append(_cache() if cache is None else cache, packed if args else None, None)


def _attend(cache=None, args=True, ws=P, wsb=1 << 40, **kw):
    a = dict(q=P, out=P, pos=P, shared=0, qs=(512, 512, 64), os=(512, 512, 64), ps=1, T=1, H=8, window=0, prefixes=0, max_len=0, scale=0.0)
    a.update(kw)
    packed = decoding._ATTEND.pack(a["q"] or 0, a["out"] or 0, a["pos"] or 0, a["shared"], *a["qs"], *a["os"], a["ps"], a["T"], a["H"], a["window"], a["prefixes"], a["max_len"],
                                   a["scale"])
    return sg.load_library().specgbv_packed_attend(_cache() if cache is None else cache, packed if args else None, ws, wsb, None)


def _read(cache=None, args=True, **kw):
    a = dict(k=P, v=P, pos=P, ks=(256, 256, 64), vs=(256, 256, 64), ps=1, T=1)
    a.update(kw)
    packed = decoding._READ.pack(a["k"] or 0, a["v"] or 0, a["pos"] or 0, *a["ks"], *a["vs"], a["ps"], a["T"], 0)
    return sg.load_library().specgbv_packed_read(_cache() if cache is None else cache, packed if args else None, None)


@pytest.mark.parametrize("call", [_append, _attend, _read])
def test_bad_caches(call):
    for change, status in BAD_CACHES:
        assert call(_cache(**change)) == status, (change, sg.specgbv_last_error())
        assert sg.specgbv_last_error()
    assert call(args=False) == 1
    assert call(_cache(S=0, table=None), T=1) == 0           # nothing to do
    assert call(T=0) == 0


def test_bad_arguments():
    for kw, status in ((dict(T=-1), 1), (dict(H=0), 1), (dict(H=6), 1), (dict(pairs=-1), 1), (dict(pairs=33), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
                       (dict(eps=float("inf")), 1), (dict(qs=(-1, 1, 1)), 1), (dict(T=2), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(out=None), 1),
                       (dict(pos=None), 1), (dict(freq=None), 1), (dict(q=P + 1), 1), (dict(pos=P + 2), 1), (dict(freq=P + 4), 1), (dict(T=1 << 30, ps=1 << 30), 2)):
        assert _append(**kw) == status, (kw, sg.specgbv_last_error())
    for kw, status in ((dict(T=-1), 1), (dict(H=0), 1), (dict(H=6), 1), (dict(window=-1), 1), (dict(max_len=-1), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1),
                       (dict(prefixes=2), 1), (dict(prefixes=-1), 1), (dict(prefixes=3), 1), (dict(os=(1, -1, 1)), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(pos=None), 1),
                       (dict(q=P + 1), 1), (dict(pos=P + 1), 1), (dict(prefixes=1, shared=P, ws=0), 3), (dict(prefixes=1, shared=P, ws=P + 8), 3),
                       (dict(prefixes=1, shared=P, wsb=64), 3)):
        assert _attend(**kw) == status, (kw, sg.specgbv_last_error())
    for kw, status in ((dict(T=-1), 1), (dict(T=2), 1), (dict(ks=(-1, 1, 1)), 1), (dict(vs=(1, 1, -1)), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(pos=None), 1),
                       (dict(k=P + 1), 1), (dict(pos=P + 2), 1)):
        assert _read(**kw) == status, (kw, sg.specgbv_last_error())


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses here are no GPU's: nothing may come to a launch")
def test_calls_that_a_launch_holds_and_that_none_holds():
    def cache(S, H, G, T):
        return _cache(S=S, G=G, kp=16 * G * 32, vp=16 * G * 32, ksp=32 * G, vsp=32 * G)
    for S, T, H, G, fits in ((2 ** 22, 1, 8, 8, True), (2 ** 23, 1, 8, 8, False)):
        big = (T * H * 64, H * 64, 64)
        assert _attend(cache(S, H, G, T), qs=big, os=big, T=T, H=H) == (4 if fits else 2), sg.specgbv_last_error()
    for S, T, H, G, fits in ((2 ** 24 - 1, 1, 8, 8, True), (2 ** 26, 1, 8, 8, False), (1, 1, 2 ** 29, 1, False)):
        big, kv = (T * H * 64, H * 64, 64), (T * G * 64, G * 64, 64)
        assert _append(cache(S, H, G, T), qs=big, os=big, ks=kv, vs=kv, T=T, H=H) == (4 if fits else 2), sg.specgbv_last_error()


def _pool(**kw):
    a = dict(table=P, ring=P, ends=P, held=P, ts=6, pages=40, page=16, B=3, K=2, width=6)
    a.update(kw)
    return decoding._POOL.pack(*[a[x] or 0 for x in "table ring ends held ts pages page B K width".split()], 0)


def _advance(pool=None, args=True, ws=P, wsb=1 << 30, **kw):
    a = dict(length=P, chosen=P, shared=P, served=P, room=0)
    a.update(kw)
    packed = decoding._ADVANCE.pack(a["length"] or 0, a["chosen"] or 0, a["shared"] or 0, a["served"] or 0, a["room"], 0)
    return sg.load_library().specgbv_pages_advance(_pool() if pool is None else pool, packed if args else None, ws, wsb, None)


def test_bad_pools():
    for kw, status in ((dict(pages=0), 1), (dict(page=0), 1), (dict(B=-1), 1), (dict(K=0), 1), (dict(width=0), 1), (dict(ts=5), 1), (dict(pages=1 << 30), 2),
                       (dict(width=1 << 20, ts=1 << 20, page=1 << 11), 2), (dict(width=1 << 15, ts=1 << 15, B=1 << 14, K=4), 2), (dict(table=None), 1), (dict(ring=None), 1),
                       (dict(ends=None), 1), (dict(held=None), 1), (dict(table=P + 2), 1), (dict(held=P + 1), 1)):
        assert _advance(_pool(**kw)) == status, (kw, sg.specgbv_last_error())
    for kw in (dict(length=None), dict(shared=None), dict(served=None), dict(room=-1), dict(length=P + 1), dict(chosen=P + 2)):
        assert _advance(**kw) == 1, (kw, sg.specgbv_last_error())
    assert _advance(args=False) == 1
    assert _advance(_pool(B=0, table=None)) == 0
    big = _pool(B=2000, width=40, ts=40)
    need = sg.load_library().specgbv_pages_workspace_bytes(big)
    assert need > 0 and sg.load_library().specgbv_pages_workspace_bytes(_pool()) == 0 and sg.load_library().specgbv_pages_workspace_bytes(_pool(K=0)) == 0
    assert _advance(big, ws=0) == 3 and _advance(big, ws=P + 8) == 3 and _advance(big, wsb=need - 1) == 3


def _slots(args=True, **kw):
    a = dict(table=P, start=P, count=P, pos=P, slots=P, ts=6, ps=5, ss=5, S=4, K=2, width=6, page=16, pages=40, T=5, right=0)
    a.update(kw)
    packed = decoding._SLOTS.pack(*[a[x] or 0 for x in "table start count pos slots ts ps ss S K width page pages T right".split()], 0)
    return sg.load_library().specgbv_slot_map(packed if args else None, None)


def test_bad_slot_maps():
    for kw, status in ((dict(S=-1), 1), (dict(K=0), 1), (dict(S=5), 1), (dict(width=0), 1), (dict(page=0), 1), (dict(pages=0), 1), (dict(T=-1), 1), (dict(ts=5), 1), (dict(ps=4), 1),
                       (dict(ss=4), 1), (dict(table=None), 1), (dict(start=None), 1), (dict(count=None), 1), (dict(pos=None), 1), (dict(pos=P + 2), 1), (dict(slots=P + 4), 1),
                       (dict(width=1 << 20, ts=1 << 20, page=1 << 11), 2), (dict(S=1 << 28, T=8, ps=8, ss=8), 2)):
        assert _slots(**kw) == status, (kw, sg.specgbv_last_error())
    assert _slots(args=False) == 1 and _slots(S=0) == 0 and _slots(T=0) == 0


class _Said(torch.Tensor):
    """A CPU tensor that says it lives on a GPU."""
    is_cuda = True


def _said(x):
    return x.as_subclass(_Said)


def _parts(S=3, width=4, pages=8, G=2, page=8, D=64):
    kv = [_said(torch.zeros((pages, G, page, D // 2), dtype=torch.uint8)) for _ in range(2)]
    scale = [_said(torch.zeros((pages, G, D // 32, page), dtype=torch.uint8)) for _ in range(2)]
    return kv + scale + [_said(torch.zeros((S, width), dtype=torch.int32))]


needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses here are no GPU's: nothing may come to a launch")


@needs_no_gpu
def test_what_a_packed_cache_is_made_of():
    k, v, ks, vs, table = _parts()
    cache = sg.PackedCache(k, v, ks, vs, table)
    assert (cache.pages, cache.kv_heads, cache.page_size, cache.head_dim, cache.sequences, cache.width, cache.dtype) == (8, 2, 8, 64, 3, 4, torch.bfloat16)
    for bad in ((k[0], v, ks, vs, table), (k, v[:4], ks, vs, table), (k, v, ks[:, :, :1], vs, table), (k, v, ks, vs.transpose(2, 3), table), (k, v, ks, vs, table[0]),
                (k, v, ks, vs, table.long()), (k.transpose(2, 3), v.transpose(2, 3), ks, vs, table), (k[..., :24], v[..., :24], ks, vs, table), (torch.zeros_like(k).as_subclass(torch.Tensor), v, ks, vs, table)):
        with pytest.raises(ValueError):
            sg.PackedCache(*bad)
    for bad in ((k.short(), v, ks, vs, table), (k, v, ks.bool(), vs, table)):
        with pytest.raises(TypeError):
            sg.PackedCache(*bad)
    with pytest.raises(TypeError):
        sg.PackedCache(k, v, ks, vs, table, torch.float16)
    with pytest.raises(ValueError):
        sg.PackedCache.empty(4, 2, 8, 40, table)


@needs_no_gpu
def test_the_stride_of_a_dimension_of_one_is_of_no_matter():
    kv = [_said(torch.zeros(4096, dtype=torch.uint8).as_strided((1, 1, 8, 16), (7, 3, 16, 1))) for _ in range(2)]
    scale = [_said(torch.zeros(4096, dtype=torch.uint8).as_strided((1, 1, 1, 8), (5, 1, 1, 1))) for _ in range(2)]
    cache = sg.PackedCache(*kv, *scale, _said(torch.zeros((0, 4), dtype=torch.int32)))
    pos = _said(torch.zeros((0, 2), dtype=torch.int32))
    assert sg.specgbv_packed_read(cache, pos, stream=0)[0].shape == (0, 2, 1, 32)
    q = _said(torch.zeros((0, 2, 4, 32), dtype=torch.bfloat16))
    assert sg.specgbv_packed_attend(cache, q, pos, stream=0)[0].shape == q.shape


@needs_no_gpu
def test_what_calls_on_a_packed_cache_look_at():
    cache = sg.PackedCache(*_parts())
    pos = _said(torch.zeros((3, 2), dtype=torch.int32))
    q, k = (_said(torch.zeros((3, 2, h, 64), dtype=torch.bfloat16)) for h in (4, 2))
    for a in ((q[:2], k, k, pos), (q, k[:, :1], k, pos), (q, k, k[..., :32], pos), (q, k, k, pos[:, :1]), (q, k, k, pos.long())):
        with pytest.raises(ValueError):
            sg.specgbv_packed_append(cache, *a, stream=0)
    with pytest.raises(TypeError):
        sg.specgbv_packed_append(cache, q.float(), k, k, pos, stream=0)
    for kw in (dict(out=q[:, :1]), dict(inv_freq=_said(torch.zeros(4))), dict(q_weight=_said(torch.zeros(63, dtype=torch.bfloat16)))):
        with pytest.raises(ValueError):
            sg.specgbv_packed_append(cache, q, k, k, pos, stream=0, **kw)
    for kw in (dict(shared_len=_said(torch.zeros(0, dtype=torch.int32))), dict(out=q[:, :1]), dict(workspace=torch.zeros(1 << 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            sg.specgbv_packed_attend(cache, q, pos, stream=0, **kw)
    with pytest.raises(sg.SpecGBVError):
        sg.specgbv_packed_attend(cache, q, pos, stream=0, window=-1)
    for kw in (dict(k=q), dict(v=k[:, :1])):
        with pytest.raises(ValueError):
            sg.specgbv_packed_read(cache, pos, stream=0, **kw)
    with pytest.raises(ValueError):
        sg.specgbv_packed_read(cache, pos[0], stream=0)
    none = sg.PackedCache(*_parts(S=0))
    assert sg.specgbv_packed_read(none, _said(torch.zeros((0, 3), dtype=torch.int32)), stream=0)[0].shape == (0, 3, 2, 64)


@needs_no_gpu
def test_a_workspace_serves_every_max_len_of_drawn_shapes():
    """What is asked for at any max_len is no more than the size that is given for all."""
    import random
    rng = random.Random(5)
    lib = sg.load_library()
    for _ in range(3000):
        G, D, T = rng.choice([1, 2, 3, 8]), rng.choice([32, 64, 96, 128, 192, 256]), rng.choice([1, 2, 5, 9, 17, 40, 100, 400])
        H, K, page = G * rng.choice([1, 2, 4, 7, 32]), rng.choice([1, 1, 2, 8]), rng.choice([8, 16, 64])
        B, width, dtype = rng.choice([1, 2, 7, 16, 33, 64, 65, 130, 300]), rng.choice([1, 3, 20, 130, 600, 5000]), rng.choice([0, 1])
        S, prefixes, window = B * K, B if K > 1 else rng.choice([0, B]), rng.choice([0, 0, 1, 90, 1500])
        cache = _cache(S=S, G=G, D=D, page=page, width=width, ts=width, dtype=dtype, kp=page * G * D // 2, kh=page * D // 2, kt=D // 2, vp=page * G * D // 2, vh=page * D // 2, vt=D // 2,
                       ksp=G * D // 32 * page, ksh=D // 32 * page, ksb=page, vsp=G * D // 32 * page, vsh=D // 32 * page, vsb=page)
        rows = dict(T=T, H=H, window=window, prefixes=prefixes, shared=P if prefixes else 0, qs=(T * H * D, H * D, D), os=(T * H * D, H * D, D), ps=T)
        packed = decoding._ATTEND.pack(P, P, P, rows["shared"], *rows["qs"], *rows["os"], T, T, H, window, prefixes, 0, 0.0)
        need = lib.specgbv_packed_attend_workspace_bytes(cache, packed)
        for n in [0] + [rng.randint(1, width * page + 5) for _ in range(12)]:
            assert _attend(cache, wsb=need, max_len=n, **rows) == 4, (n, need, rows, B, K, G, D, page, width, dtype, sg.specgbv_last_error())         # (no GPU: it comes to the launch)


@needs_no_gpu
@pytest.mark.parametrize("prefixes,drafts", [(1, 1), (4, 8), (70, 1), (70, 2), (300, 1)])
@pytest.mark.parametrize("window", [0, 700])
def test_a_workspace_serves_every_max_len(prefixes, drafts, window):
    for G, D, T, heads, dtype in ((8, 128, 8, 32, torch.bfloat16), (8, 128, 1, 32, torch.bfloat16), (1, 64, 1, 5, torch.float32), (2, 256, 9, 8, torch.bfloat16), (1, 64, 40, 8, torch.float32)):
        S = prefixes * drafts
        for shared in ([None, _said(torch.zeros(prefixes, dtype=torch.int32))] if drafts > 1 else [None]):
            parts = _parts(S=S, width=600, pages=1, G=G, D=D)
            cache = sg.PackedCache(*parts, dtype)
            q = _said(torch.zeros((1, 1, 1, 1), dtype=dtype).expand(S, T, heads, D).contiguous())
            need = {n: sg.specgbv_packed_attend_workspace_bytes(cache, q, window=window, shared_len=shared, max_len=n) for n in (0, 1, 40, 208, 209, 513, 1024, 4000, 1 << 20)}
            assert len(set(need.values())) == 1, (G, D, T, shared is None, need)
            for n in need:                                   # (no GPU: it comes to the launch)
                args = decoding._attend_args(cache, q, q.stride(), T, heads, P, q.stride(), P, T, window, shared, n, None)
                assert sg.load_library().specgbv_packed_attend(cache._c, args, P, max(need[n], 256), None) == 4, (n, sg.specgbv_last_error())


@needs_no_gpu
def test_what_a_pool_and_a_slot_map_look_at():
    table, ring = _said(torch.zeros((6, 4), dtype=torch.int32)), _said(torch.zeros(20, dtype=torch.int32))
    ends, held = _said(torch.zeros(2, dtype=torch.int32)), _said(torch.zeros((3, 2), dtype=torch.int32))
    pool = sg.PagePool(table, ring, ends, held, drafts=2, page_size=8)
    assert (pool.prefixes, pool.drafts, pool.width, pool.pages) == (3, 2, 4, 20)
    for a, kw in (((table[0], ring, ends, held), {}), ((table.long(), ring, ends, held), {}), ((table, ring[::2], ends, held), {}), ((table, ring, ring, held), {}),
                  ((table, ring, ends, held[:2]), {}), ((table, ring, ends, held), dict(drafts=4)), ((table, ring, ends, held), dict(drafts=0)),
                  ((table.as_subclass(torch.Tensor), ring, ends, held), {}), ((table.t(), ring, ends, held), dict(drafts=1))):
        with pytest.raises(ValueError):
            sg.PagePool(*a, **dict(dict(drafts=2, page_size=8), **kw))
    length = _said(torch.zeros(3, dtype=torch.int32))
    for kw in (dict(length=length[:2]), dict(length=length.long()), dict(chosen=length[:1]), dict(shared_len=length.float()), dict(served=_said(torch.zeros((3, 2), dtype=torch.int32))[:, 0]),
               dict(workspace=torch.zeros(256, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            sg.specgbv_pages_advance(pool, kw.pop("length", length), stream=0, **kw)
    with pytest.raises(sg.SpecGBVError):
        sg.specgbv_pages_advance(pool, length, room=-1, stream=0)
    start = _said(torch.zeros(3, dtype=torch.int32))
    for t, s, c, kw in ((table, start[:2], start, {}), (table, start, start.long(), {}), (table, start, start, dict(drafts=4)), (table, start, start, dict(tokens=-1)),
                        (table.long(), start, start, {}), (table, start, start, dict(positions=start)), (table, start, start, dict(slots=_said(torch.zeros((6, 5), dtype=torch.int32))))):
        with pytest.raises(ValueError):
            sg.specgbv_slot_map(t, s, c, **dict(dict(tokens=5, page_size=8, pages=20, drafts=2, stream=0), **kw))
    with pytest.raises(sg.SpecGBVError):
        sg.specgbv_slot_map(table, start, start, 5, page_size=0, pages=20, drafts=2, stream=0)
    positions, slots = sg.specgbv_slot_map(table, start, start, 0, page_size=8, pages=20, drafts=2, stream=0)
    assert positions.shape == (6, 0) and slots.shape == (6, 0)
