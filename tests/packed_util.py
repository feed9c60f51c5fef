"""Caches held in 4 bits, plain float64 references and error bounds for the tests of the operators on them."""
import math

import numpy as np

from decoding_util import HALF_STEP, host, torch_dtype

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BORDERS = (SIZES[1:] + SIZES[:-1]) / 2
CODES = np.concatenate((SIZES, -SIZES))


def quantise(y):
    """(codes, scale bytes) of float64 values [..., D], from the definition."""
    x = y.reshape(y.shape[:-1] + (-1, 32))
    odd = ~np.isfinite(x).all(-1)
    x = np.where(np.isfinite(x), x, 0.0)
    most = np.abs(x).max(-1)
    e = np.full(most.shape, -120)
    for n in range(-119, 126):
        e = np.where(most > 7.0 * 2.0 ** (n - 1), n, e)
    t = np.abs(x) * 2.0 ** -e.astype(np.float64)[..., None]
    below, above = np.searchsorted(BORDERS, t, side="left"), np.searchsorted(BORDERS, t, side="right")
    code = np.where(below % 2 == 0, below, above) + 8 * np.signbit(x)
    code = np.where(odd[..., None], 0, code)
    return code.reshape(y.shape).astype(np.uint8), np.where(odd, 255, e + 127).astype(np.uint8)


def values(code, byte):
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127.0))
    return CODES[code] * np.repeat(scale, 32, axis=-1)


def pack(code):
    return (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)


def unpack(data):
    out = np.empty(data.shape[:-1] + (2 * data.shape[-1],), np.uint8)
    out[..., 0::2], out[..., 1::2] = data & 15, data >> 4
    return out


def make_packed(gen, S, width, page, G, D, dtype="bf16", token_major=False, extra=3, spread=3, page_stride=None):
    """A PackedCache on the GPU of random codes and of powers of two around 1; pages dealt out in random order."""
    import torch

    import paper_2604_25925_amd as sg
    dev = torch.device("cuda")
    pages = S * width + extra
    table = torch.from_numpy(gen.permutation(pages)[:S * width].astype(np.int32).reshape(S, width)).to(dev)
    data = []
    for _ in range(2):
        x = torch.from_numpy(gen.integers(0, 256, (pages, page, G, D // 2) if token_major else (pages, G, page, D // 2), dtype=np.uint8)).to(dev)
        x = x.transpose(1, 2) if token_major else x
        if page_stride is not None:                           # pages far apart
            room = torch.zeros((pages - 1) * page_stride + G * page * D // 2, dtype=torch.uint8, device=dev)
            far = room.as_strided(x.shape, (page_stride,) + (x.stride() if not token_major else x.stride())[1:])
            far.copy_(x)
            x = far
        data.append(x)
    scales = [torch.from_numpy(gen.integers(127 - spread, 127 + 1, (pages, G, D // 32, page), dtype=np.uint8)).to(dev) for _ in range(2)]
    return sg.PackedCache(data[0], data[1], scales[0], scales[1], table, torch_dtype(dtype))


def dense(cache):
    """(k, v) of a cache as float64 [pages, G, page, D] on the host."""
    both = np.stack((CODES[np.arange(256) & 15], CODES[np.arange(256) >> 4]), axis=-1)         # of a byte
    out = []
    for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x, byte = x.cpu().numpy(), np.swapaxes(s.cpu().numpy(), 2, 3)
        scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127.0))
        out.append((both[x].reshape(x.shape[:3] + (-1, 32)) * scale[..., None]).reshape(x.shape[:3] + (-1,)))
    return out


def plain_attend(cache, q, positions, window=0, scale=None, table=None):
    """(out, sums of the weights times values' magnitudes, bounds of the weights' relative errors) in float64, query by query."""
    k, v = dense(cache)
    q, positions = host(q), positions.cpu().numpy()
    table = cache.table.cpu().numpy() if table is None else table
    S, T, H, D = q.shape
    pages, G, P, _ = k.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, mass, wobble = np.zeros(q.shape), np.zeros(q.shape), np.zeros((S, T, H, 1))
    for s in range(S):
        for t in range(T):
            pos = min(int(positions[s, t]), table.shape[1] * P - 1)
            lo = max(0, int(positions[s, t]) - window + 1) if window > 0 else 0
            at = np.arange(lo, pos + 1)
            if at.size:
                at = at[(table[s, at // P] >= 0) & (table[s, at // P] < pages)]
            if not at.size:
                continue
            pg, sl = table[s, at // P], at % P
            for g in range(G):
                kk, vv = k[pg, g, sl], v[pg, g, sl]
                rows = slice(g * (H // G), (g + 1) * (H // G))
                x = q[s, t, rows] @ kk.T * scale
                with np.errstate(invalid="ignore"):
                    w = np.exp(x - x.max(-1, keepdims=True))
                    w /= w.sum(-1, keepdims=True)
                    out[s, t, rows] = w @ vv
                    mass[s, t, rows] = w @ np.abs(vv)
                    # a score: D products, whose sums the matrix instructions may cut off instead of rounding, and the scaling; a weight: its exponential
                    wobble[s, t, rows, 0] = (D + 8) * 2.0 ** -23 * np.max(np.abs(q[s, t, rows]) @ np.abs(kk).T, axis=-1) * abs(scale) + (len(at) + 64) * 2.0 ** -23
    return out, mass, wobble


def bound(out, mass, wobble, dtype):
    """A weight is off by the exponential of its score's error (numerator and denominator: twice) and, with bfloat16, by a rounding for the product;
    the result is rounded once."""
    half = HALF_STEP[dtype]
    return half * np.abs(out) + mass * (2 * wobble + (half if dtype == "bf16" else 0.0)) * (1 + half) + 1e-30


def check(got, cache, q, positions, dtype, window=0, scale=None, label=""):
    ref, mass, wobble = plain_attend(cache, q, positions, window, scale)
    g = host(got)
    assert np.all(np.isfinite(g)), label + ": not finite"
    off = np.abs(g - ref) / bound(ref, mass, wobble, dtype)
    assert off.max(initial=0.0) <= 1.0, "%s: %.3g times the bound at %s" % (label, off.max(), np.unravel_index(off.argmax(), off.shape))
    return ref
