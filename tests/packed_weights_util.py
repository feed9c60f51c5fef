"""Caches of 4 bits of known codes; among them such whose attention gives the weights themselves, in float32: `live` keys with one entry of 1 each, so that a score is one entry of the query, and
values with one entry of 1 each, so that a result's entries are the weights; all other keys meet an entry of the query that leaves their weight 0."""
import numpy as np

from packed_util import make_packed, pack

ONE = 2                                                       # the code of 1
WAYS = {"one pass": (3, 2, 90), "filled": (40, 2, 1060), "parts": (2, 1, 2500), "waves": (265, 4, 60)}       # sequences, kv heads, tokens: how a call is cut
LIVE = 24
RANGE = 3.0                                                   # scores lie in [-RANGE, RANGE]


def queries(gen, shape):
    """Entry 0 makes a weight of 0; entries 1 to LIVE are the scores of the live keys.  All 24 bits of each are of matter."""
    q = np.zeros(shape, np.float32)
    q[..., 0] = -2000.0
    q[..., 1:1 + LIVE] = gen.uniform(-RANGE, RANGE, shape[:-1] + (LIVE,))
    return q


def weights(q):
    """The weights of the live keys in float64, for a scale of 1."""
    x = q[..., 1:1 + LIVE].astype(np.float64)
    w = np.exp(x - x.max(-1, keepdims=True))
    return w / w.sum(-1, keepdims=True)


def bound():
    """Largest relative error of a weight held in 24 bits.  A score's product is exact (one entry of 1), its scaling, which the reference is taken from at once,
    one rounding of at most 2 RANGE log2(e) + 8 (a reference is raised where a score is 8 above it), the scale's own another of the same; both in the exponent, twice for numerator and
    denominator.  An exponential: two steps; the sums of LIVE weights and of zeros, LIVE roundings at most; the parts' and waves' factors, two exponentials and two
    products; quotient and product one each."""
    exponent = 2 * RANGE * 1.4426950408889634 + 8
    return (2 * 2 * exponent * np.log(2.0) + 2 * 2 + LIVE + 2 * 4 + 2) * 2.0 ** -24


def cut(x, operands):
    """Floats as the sum of so many bfloat16 values, each cut off."""
    out, rest = np.zeros(x.shape, np.float32), x.astype(np.float32)
    for _ in range(operands):
        part = (rest.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
        out, rest = out + part, rest - part
    return out


def emulated(q, of_queries, of_weights):
    """The weights where queries and weights are the sums of so many operands."""
    x = cut(q[..., 1:1 + LIVE], of_queries).astype(np.float64)
    w = np.exp(x - x.max(-1, keepdims=True)).astype(np.float32)
    return cut(w, of_weights).astype(np.float64) / w.astype(np.float64).sum(-1, keepdims=True)


def zero_cache(gen, S, width, page, G, D, dtype):
    """A cache of zeros with powers of 1."""
    cache = make_packed(gen, S, width, page, G, D, dtype)
    for x in (cache.k, cache.v):
        x.zero_()
    for x in (cache.k_scale, cache.v_scale):
        x.fill_(127)
    return cache


def put_codes(cache, name, where, rows):
    """Codes [S, tokens, G, D] of a sequence's tokens at positions where [S, tokens]."""
    import torch
    data, table = getattr(cache, name).cpu().numpy(), cache.table.cpu().numpy()
    packed = pack(rows)
    for s in range(where.shape[0]):
        at = where[s]
        data[table[s, at // cache.page_size], :, at % cache.page_size] = packed[s]
    getattr(cache, name).copy_(torch.from_numpy(data))
