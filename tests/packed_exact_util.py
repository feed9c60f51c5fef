"""What a packed cache has to hold after an append, entry by entry: keys normalised and turned in more than float64, and the codes that the
kernel's own error leaves open."""
from decimal import Decimal, getcontext

import numpy as np

from decoding_util import host, torch_dtype
from packed_util import BORDERS, pack

getcontext().prec = 80
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def on_gpu(x, dtype="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(torch_dtype(dtype))


def marked_cache(table, pages, page, G, D, dtype):
    """A cache whose every byte is 0xA5, and its bytes (data, scale) by name."""
    import torch

    import paper_2604_25925_amd as sg
    data = [torch.full((pages, G, page, D // 2), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.full((pages, G, D // 32, page), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = sg.PackedCache(*data, *scale, table, torch_dtype(dtype))
    return cache, {n: (getattr(cache, n).cpu().numpy(), getattr(cache, n + "_scale").cpu().numpy()) for n in ("k", "v")}


def turns(positions, inv_freq):
    """(cos, sin) of positions [...] times float64 frequencies [R] as longdouble [..., R]: the product and its remainder by 2 pi in 80 digits."""
    p = np.asarray(positions)
    angle = np.empty(p.shape + (len(inv_freq),), np.longdouble)
    for i in np.ndindex(p.shape):
        for r, f in enumerate(inv_freq):
            x = Decimal(int(p[i])) * Decimal(float(f))
            x -= 2 * PI * (x / (2 * PI)).to_integral_value()
            angle[i + (r,)] = np.longdouble(float(x)) + np.longdouble(float(x - Decimal(float(x))))
    return np.cos(angle), np.sin(angle)


def turned(x, positions, inv_freq, weight=None, eps=0.0, interleaved=False):
    """Heads [S, T, G, D] normalised and turned, as longdouble, and how far the kernel's float64 may be from each entry.

    The turn: 1 / (2 pi) and the product have tails, so half a step of the remaining quarter to half turn, 2^-55, is 2^-52.3 of an angle; the sine and
    cosine are at most 4 steps of 2^-53 off, and the two products and the sum two roundings: below 2^-50 (|a| + |b|) for a pair (a, b).  The norm: a sum of D squares (8 in a lane,
    then at most 5 exchanges), its mean and eps count half behind the root, and the root, its reciprocal and two products one each: 11.5 roundings of 2^-53,
    below 2^-49.  What neither turns nor is normalised is exact, and so is what turns by 0."""
    y = host(x).astype(np.longdouble)
    off = np.zeros(y.shape, np.longdouble)
    if weight is not None:
        y = y * host(weight).astype(np.longdouble) / np.sqrt((y * y).mean(-1, keepdims=True) + np.longdouble(eps))
        off = np.abs(y) * 2.0 ** -49
    R = 0 if inv_freq is None else len(inv_freq)
    if R:
        cos, sin = (z[:, :, None] for z in turns(np.maximum(positions, 0), inv_freq))
        a, b = (slice(0, 2 * R, 2), slice(1, 2 * R, 2)) if interleaved else (slice(0, R), slice(R, 2 * R))
        mass = np.abs(y[..., a]) + np.abs(y[..., b])
        out = y.copy()
        out[..., a], out[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
        turning = (np.asarray(positions) > 0)[..., None, None]
        norm_off = mass * 2.0 ** -49 if weight is not None else 0.0 * mass
        off = off.copy()
        off[..., a] = off[..., b] = norm_off + np.where(turning, mass * 2.0 ** -50, 0.0)
        y = out
    return y, off


def power(most):
    """The scale byte of blocks whose largest magnitude is `most` (finite)."""
    e = np.full(most.shape, -120)
    for n in range(-119, 126):
        e = np.where(most > np.longdouble(7.0) * np.longdouble(2.0) ** (n - 1), n, e)
    return e + 127


def code(y, byte):
    """Codes of entries [..., D] in blocks of the given powers."""
    t = np.abs(y) * np.repeat(np.longdouble(2.0) ** (127 - byte.astype(np.int64)).astype(np.longdouble), 32, axis=-1)
    below, above = np.searchsorted(BORDERS, t, side="left"), np.searchsorted(BORDERS, t, side="right")
    return (np.where(below % 2 == 0, below, above) + 8 * np.signbit(y)).astype(np.uint8)


def check_bytes(cache, name, before, y, off, positions, label=""):
    """Every byte of k or v and its scales: those of tokens [S, T] at positions as y says, all others as in `before` (data, scale).  Where an entry's error `off` reaches over
    a border it may have one of the two codes there, where the largest of a block's reaches over a power's, the block may have one of the two."""
    data, scale = getattr(cache, name).cpu().numpy(), getattr(cache, name + "_scale").cpu().numpy()
    want, want_scale = before[0].copy(), before[1].copy()
    table = cache.table.cpu().numpy()
    page_size, open_entries = cache.page_size, 0
    for s, t in np.ndindex(positions.shape):
        n = int(positions[s, t])
        if n < 0 or n >= table.shape[1] * page_size or not 0 <= table[s, n // page_size] < cache.pages:
            continue
        at = int(table[s, n // page_size])
        got = scale[at, :, :, n % page_size]
        x, err = y[s, t], off[s, t]
        size, blocks = np.abs(x), x.shape[:-1] + (-1, 32)
        lo, hi = power(np.maximum(size - err, 0).reshape(blocks).max(-1)), power((size + err).reshape(blocks).max(-1))
        assert ((got == lo) | (got == hi)).all(), (label, name, "power", s, t)
        first, last = (code(np.where(err > 0, z, x), got) for z in (x - err, x + err))         # (-0 + 0 has another sign)
        bytes_got = data[at, :, n % page_size]
        codes = np.stack((bytes_got & 15, bytes_got >> 4), axis=-1).reshape(x.shape)
        wrong = (codes != first) & (codes != last)
        assert not wrong.any(), (label, name, "code", s, t, np.argwhere(wrong)[:4].tolist())
        open_entries += int((first != last).sum())
        want_scale[at, :, :, n % page_size] = got
        want[at, :, n % page_size] = pack(codes)
    assert (data == want).all() and (scale == want_scale).all(), (label, name, "bytes that no token has")
    return open_entries
