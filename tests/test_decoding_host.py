"""CPU-only checks of the decoding step's operators: the layout of their C structures, every refusal that the host makes before a
launch, and where a token lives for tables with pages that are not there (the kernels' own functions, compiled for the host)."""
import ctypes
import os
import re
import shutil
import struct
import subprocess

import pytest

import paper_2604_25925_amd as sg
from paper_2604_25925_amd import decoding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                                  # an address that is never looked at: every call is refused before

CACHE_FIELDS = ("k v table k_page_stride k_head_stride k_token_stride v_page_stride v_head_stride v_token_stride table_stride pages "
                "kv_heads page_size head_dim sequences table_width dtype reserved").split()
APPEND_FIELDS = ("q k v q_out positions inv_freq q_weight k_weight q_stride k_stride v_stride q_out_stride positions_stride eps tokens "
                 "heads pairs interleaved").split()
ATTEND_FIELDS = "q out positions shared_len q_stride out_stride positions_stride tokens heads window prefixes max_len scale".split()


def test_packed_arguments_have_the_c_structures_layout(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    items = (("specgbv_paged_cache", decoding._CACHE, CACHE_FIELDS), ("specgbv_append_args", decoding._APPEND, APPEND_FIELDS),
             ("specgbv_attend_args", decoding._ATTEND, ATTEND_FIELDS))
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "%s"' % os.path.join(ROOT, "include", "specgbv.h"), 'int main(void) {']
    for name, _, fields in items:
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        for f in fields:
            lines.append('printf("%s.%s %%zu %%zu\\n", offsetof(%s, %s), sizeof(((%s *)0)->%s));' % (name, f, name, f, name, f))
    (tmp_path / "layout.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run([cc, "-std=c99", "-o", str(tmp_path / "layout"), str(tmp_path / "layout.c")], check=True)
    got = dict(l.split(" ", 1) for l in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines())
    header = open(os.path.join(ROOT, "include", "specgbv.h")).read()
    for name, packer, fields in items:
        assert int(got[name]) == packer.size, name
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, header).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        declared = [re.sub(r"\[\d+\]|\W", "", x) for d in body.split(";") if d.strip() for x in re.sub(r"^\s*(const\s+)?\w+", "", d.strip()).split(",")]
        assert declared == fields, name
        at = 0                                               # no gaps: the packed order is the declared one
        for f in fields:
            offset, size = map(int, got["%s.%s" % (name, f)].split())
            assert offset == at, (name, f)
            at += size
        assert at == packer.size


def _cache(**kw):
    a = dict(k=P, v=P, table=P, kp=4096, kh=1024, kt=64, vp=4096, vh=1024, vt=64, ts=5, pages=9, G=4, page=16, D=64, S=3, width=5, dtype=1)
    a.update(kw)
    return decoding._CACHE.pack(a["k"], a["v"], a["table"], a["kp"], a["kh"], a["kt"], a["vp"], a["vh"], a["vt"], a["ts"], a["pages"],
                                a["G"], a["page"], a["D"], a["S"], a["width"], a["dtype"], 0)


BAD_CACHES = [(dict(dtype=2), 1), (dict(pages=0), 1), (dict(G=0), 1), (dict(S=-1), 1), (dict(width=0), 1), (dict(page=0), 1), (dict(D=0), 1),
              (dict(D=60), 2), (dict(D=264), 2), (dict(page=12), 2), (dict(width=1 << 20, ts=1 << 20, page=1 << 11), 2), (dict(ts=4), 1),
              (dict(kt=-64), 1), (dict(kt=68), 2), (dict(vh=1 << 31), 2), (dict(k=None), 1), (dict(v=None), 1), (dict(table=None), 1),
              (dict(k=P + 8), 2), (dict(v=P + 8), 2), (dict(table=P + 2), 1)]


def _bytes(values, fmt):
    return struct.Struct(fmt).pack(*[0 if v is None else v for v in values])


def _append(cache=None, null_args=False, **kw):
    lib = sg.load_library()
    a = dict(q=P, k=P, v=P, out=P, pos=P, freq=P, qw=0, kw=0, qs=(512, 512, 64), ks=(256, 256, 64), vs=(256, 256, 64), os=(512, 512, 64),
             ps=1, eps=1e-6, T=1, H=8, pairs=32, inter=0)
    a.update(kw)
    args = decoding._APPEND.pack(a["q"], a["k"], a["v"], a["out"], a["pos"], a["freq"], a["qw"], a["kw"], *a["qs"], *a["ks"], *a["vs"],
                                 *a["os"], a["ps"], a["eps"], a["T"], a["H"], a["pairs"], a["inter"])
    return lib.specgbv_cache_append(_cache() if cache is None else cache, None if null_args else args, None)


def _cache_or_none(kw):
    return _cache(**{k: 0 if v is None else v for k, v in kw.items()})


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_bad_caches_are_refused(kw, status):
    lib = sg.load_library()
    assert _append(_cache_or_none(kw)) == status and sg.specgbv_last_error()
    assert _attend(_cache_or_none(kw)) == status and sg.specgbv_last_error()
    if not any(n in kw for n in ("k", "v", "table")):
        assert lib.specgbv_attend_workspace_bytes(_cache_or_none(kw), _attend_args()) == 0


def test_append_refusals():
    assert _append(null_args=True) == 1
    assert sg.load_library().specgbv_cache_append(None, None, None) == 1
    for kw in (dict(T=-1), dict(H=0), dict(H=6), dict(ps=1, T=2), dict(pairs=-1), dict(pairs=33), dict(eps=-1.0), dict(eps=float("nan")),
               dict(qs=(512, 512, -64)), dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(pos=0), dict(freq=0), dict(q=P + 1), dict(freq=P + 4),
               dict(pos=P + 2), dict(kw=P + 1)):
        assert _append(**kw) == 1, kw
        assert sg.specgbv_last_error()
    assert _append(H=1 << 20, T=1 << 20, ps=1 << 20) == 2
    assert _append(T=0) == 0 and _append(_cache(S=0)) == 0   # nothing to do


def _attend_args(**kw):
    a = dict(q=P, out=P, pos=P, shared=0, qs=(512, 512, 64), os=(512, 512, 64), ps=1, T=1, H=8, window=0, prefixes=0, max_len=0, scale=0.0)
    a.update(kw)
    return decoding._ATTEND.pack(a["q"], a["out"], a["pos"], a["shared"], *a["qs"], *a["os"], a["ps"], a["T"], a["H"], a["window"],
                                 a["prefixes"], a["max_len"], a["scale"])


def _attend(cache=None, ws=P, wsb=1 << 30, **kw):
    return sg.load_library().specgbv_attend_paged(_cache() if cache is None else cache, _attend_args(**kw), ws, wsb, None)


def test_attend_refusals():
    assert sg.load_library().specgbv_attend_paged(_cache(), None, P, 1 << 30, None) == 1
    for kw in (dict(T=-1), dict(H=0), dict(H=6), dict(ps=1, T=2), dict(window=-1), dict(max_len=-1), dict(scale=-1.0), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(prefixes=2, shared=P), dict(prefixes=-1), dict(prefixes=3), dict(q=0), dict(out=0), dict(pos=0),
               dict(q=P + 1), dict(pos=P + 2), dict(prefixes=3, shared=P + 1), dict(os=(512, -512, 64))):
        assert _attend(**kw) == 1, kw
        assert sg.specgbv_last_error()
    assert _attend(T=0) == 0 and _attend(_cache(S=0)) == 0
    # drafts of a prefix are joined over a workspace
    need = sg.load_library().specgbv_attend_workspace_bytes(_cache(), _attend_args(prefixes=1, shared=P))
    assert need > 0 and need % 256 == 0
    assert _attend(prefixes=1, shared=P, ws=None) == 3 and "need" in sg.specgbv_last_error()
    assert _attend(prefixes=1, shared=P, ws=P + 8) == 3
    assert _attend(prefixes=1, shared=P, wsb=need - 1) == 3


def test_filter_refusals():
    lib = sg.load_library()

    def call(z=P, stride=100, rows=2, V=100, dt=1, T=P, k=P, p=P, m=P, u=P, out=P, kept=P, ks=100):
        return lib.specgbv_sample_filtered(z, stride, rows, V, dt, T, k, p, m, u, out, kept, ks, P, 1 << 30, None)
    for kw in (dict(rows=-1), dict(V=0), dict(dt=5), dict(z=None), dict(out=None, kept=None), dict(u=None), dict(stride=99), dict(ks=99),
               dict(z=P + 1), dict(kept=P + 1), dict(T=P + 2), dict(k=P + 2), dict(p=P + 1), dict(m=P + 1), dict(u=P + 1), dict(out=P + 1)):
        assert call(**kw) == 1, kw
        assert sg.specgbv_last_error()
    assert call(V=(1 << 20) + 1, stride=1 << 21, ks=1 << 21) == 2
    assert call(rows=0) == 0


def test_tensors_are_checked():
    import torch
    k = torch.zeros((4, 2, 16, 64))
    with pytest.raises(ValueError):
        sg.PagedCache(k, k, torch.zeros((2, 2), dtype=torch.int32))           # not on a GPU
    with pytest.raises(TypeError):
        sg.PagedCache(k.half(), k.half(), torch.zeros((2, 2), dtype=torch.int32))
    with pytest.raises(ValueError):
        sg.PagedCache(k, k[:, :1], torch.zeros((2, 2), dtype=torch.int32))
    with pytest.raises(ValueError):
        sg.PagedCache(k, k, torch.zeros((2, 2), dtype=torch.int64))
    with pytest.raises(ValueError):
        sg.specgbv_sample_filtered(torch.zeros((2, 8)), torch.zeros(2))
    with pytest.raises(TypeError):
        sg.specgbv_sample_filtered(torch.zeros((2, 8), dtype=torch.float16), torch.zeros(2))


PLACES = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "%s"
using namespace specgbv;
static int bad(const char *what, long a, long b) { std::printf("%%s %%ld %%ld\n", what, a, b); return 1; }
int main()
{
    std::srand(7);
    const int ds[] = {1, 2, 3, 5, 7, 8, 16, 24, 40, 64, 100, 128, 1000, 4096, 65535, 65536, 1 << 20, (1 << 30) - 1, 1 << 30, 2147483647};
    for (int d : ds) {
        const Divider v = Divider::of(d);
        for (long i = 0; i < 20000; ++i) {
            long n = i < 200 ? i : i < 400 ? 2147483647L - (i - 200) : i < 10000 ? (long)(i - 5000) * d + (i %% 3) - 1 : ((long)std::rand() << 16 ^ std::rand()) & 2147483647L;
            if (n < 0 || n > 2147483647L) continue;
            const int q = v.div((int)n);
            if (q != n / d || v.mod((int)n, q) != n %% d) return bad("quotient", n, d);
        }
    }
    // tables with pages that are not there: the table is read inside its bounds only (it is as long as it says, so a sanitizer
    // sees a read behind it), and a place is inside the cache or none
    for (int round = 0; round < 300; ++round) {
        const int page = 8 * (1 + std::rand() %% 20), width = 1 + std::rand() %% 9, S = 1 + std::rand() %% 4, pages = 1 + std::rand() %% 12, stride = width + std::rand() %% 3;
        std::vector<int32_t> table((S - 1) * stride + width);
        for (int32_t &t : table) t = std::rand() %% 5 == 0 ? (std::rand() %% 2 ? -1 - std::rand() %% 100 : pages + std::rand() %% 100) : std::rand() %% pages;
        if (round %% 7 == 0) table[0] = INT32_MIN;
        if (round %% 11 == 0) table[0] = INT32_MAX;
        const PageMap m{table.data(), stride, Divider::of(page), pages, width};
        if (capacity_of(m) != (int64_t)width * page) return bad("capacity", width, page);
        for (int s = 0; s < S; ++s)
            for (long pos = -3; pos < (long)width * page + 3 * page; ++pos) {
                const Place at = place_of(m, s, (int)pos);
                const bool in = pos >= 0 && pos < (long)width * page;
                const int32_t want = in ? table[s * stride + pos / page] : -1;
                if ((at.page >= 0) != (in && want >= 0 && want < pages)) return bad("there", s, pos);
                if (at.page >= 0 && (at.page != want || at.slot != pos %% page)) return bad("place", s, pos);
                if (at.slot < 0 || at.slot >= page) return bad("slot", s, pos);
            }
        const int far[] = {2147483647, 2147483646, 1 << 30};
        for (int pos : far) if (place_of(m, S - 1, pos).page >= 0) return bad("far", pos, 0);
    }
    std::printf("ok\n");
    return 0;
}
"""


def test_places_of_tokens_with_bad_pages(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src = tmp_path / "places.cpp"
    src.write_text(PLACES % os.path.join(ROOT, "paper_2604_25925_amd", "csrc", "specgbv_paged.hpp"))
    subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-o", str(tmp_path / "places"), str(src)],
                   check=True)
    r = subprocess.run([str(tmp_path / "places")], capture_output=True, text=True, env=dict(os.environ, LD_PRELOAD=""))
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_filter_refuses_more_rows_than_a_launch_holds():
    lib = sg.load_library()
    assert lib.specgbv_sample_filtered(P, 100, 1 << 22, 100, 1, None, None, None, None, P, P, None, 100, None, 0, None) == 2
    assert "rows" in sg.specgbv_last_error()
