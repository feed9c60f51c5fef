"""CPU-only: the bound that the tests of float32 operands hold results to is one that two operands break and three keep."""
import numpy as np
import pytest

from packed_weights_util import bound, emulated, queries, weights


@pytest.mark.parametrize("seed", range(5))
def test_two_operands_exceed_the_bound_and_three_keep_it(seed):
    q = queries(np.random.default_rng(seed), (3, 4, 32))
    want = weights(q)

    def off(*operands):
        return np.abs(emulated(q, *operands) / want - 1).max()

    assert off(3, 3) < bound() / 16
    assert off(2, 3) > 4 * bound()
    assert off(3, 2) > 3 * bound()
    assert off(2, 2) > 4 * bound()
