"""Paged caches, plain float64 references and error bounds for the tests of the decoding step's operators."""
import math

import numpy as np

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # largest relative rounding error of the type


def torch_dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def make_cache(gen, S, width, page, G, D, dtype, token_major=False, extra=3, fill=None):
    """(k, v, table) on the GPU; pages dealt out in random order; `fill`: value of the whole cache instead of random ones."""
    import torch
    dev = torch.device("cuda")
    pages = S * width + extra
    table = torch.from_numpy(gen.permutation(pages)[:S * width].astype(np.int32).reshape(S, width)).to(dev)
    shape = (pages, page, G, D) if token_major else (pages, G, page, D)
    kv = []
    for _ in range(2):
        x = torch.from_numpy(gen.normal(0, 1, shape).astype(np.float32)).to(dev).to(torch_dtype(dtype)) if fill is None else \
            torch.full(shape, fill, dtype=torch_dtype(dtype), device=dev)
        kv.append(x.transpose(1, 2) if token_major else x)
    return kv[0], kv[1], table


def host(x):
    import torch
    return x.detach().to(torch.float64).cpu().numpy()


def plain_attend(q, k, v, table, positions, window=0, scale=None):
    """(out, bound of the weights' absolute sums, largest score error factor) in float64, query by query."""
    q, k, v, table, positions = host(q), host(k), host(v), table.cpu().numpy(), positions.cpu().numpy()
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
            for h in range(H):
                g = h // (H // G)
                kk, vv = k[pg, g, sl], v[pg, g, sl]
                x = kk @ q[s, t, h] * scale
                w = np.exp(x - x.max())
                w /= w.sum()
                out[s, t, h] = w @ vv
                mass[s, t, h] = w @ np.abs(vv)
                wobble[s, t, h] = (D + 4) * 2.0 ** -24 * np.max(np.abs(kk) @ np.abs(q[s, t, h])) * abs(scale) + (len(at) + 64) * 2.0 ** -24
    return out, mass, wobble


def attend_bound(out, mass, wobble, dtype):
    """Each score is off by (D + 4) half steps of float32 of its terms' absolute sum, a weight by twice that relatively, and by a
    rounding of the type for the product; the result is rounded once.  Sums of n terms: n half steps of float32."""
    half = HALF_STEP[dtype]
    return half * np.abs(out) + mass * (2 * wobble + (half if dtype == "bf16" else 0.0)) * (1 + half) + 1e-30


def check_attend(got, q, k, v, table, positions, dtype, window=0, scale=None, label=""):
    ref, mass, wobble = plain_attend(q, k, v, table, positions, window, scale)
    g = host(got)
    assert np.all(np.isfinite(g)), label + ": not finite"
    off = np.abs(g - ref) / attend_bound(ref, mass, wobble, dtype)
    assert off.max(initial=0.0) <= 1.0, "%s: %.3g times the bound at %s" % (label, off.max(), np.unravel_index(off.argmax(), off.shape))
    return ref


def plain_filter(z, T=None, top_k=None, top_p=None, min_p=None, u=None):
    """(token, kept mask) of one row of float32 values, from the definition in float64."""
    z = z.astype(np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    T = 1.0 if T is None else float(T)
    order = np.argsort(-z, kind="stable")
    order = order[z[order] > -np.inf]
    kept = np.zeros(z.size, bool)
    if order.size == 0:
        return -1, kept
    if not T > 0:
        order, T = order[:1], 1.0
    top = z[order[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(z[order] == top, 1.0, np.exp((z[order] - top) / T))
    n = order.size
    if top_k is not None and top_k > 0:
        n = min(n, int(top_k))
    if min_p is not None and min_p > 0:
        n = min(n, int((w >= min(float(min_p), 1.0)).sum()))
    w = w[:n]
    if top_p is not None and top_p < 1:
        run = np.cumsum(w)
        n = max(1, min(n, int((run - w < float(top_p) * run[-1]).sum())))
        w = w[:n]
    kept[order[:n]] = True
    if u is None:
        return None, kept
    run = np.cumsum(w)
    return int(order[min(int((run <= float(u) * run[-1]).sum()), n - 1)]), kept
