"""Attention over PC_MX4 caches where many keys of small probabilities matter beside few of large ones whose values are zero (a sink, say): against 64
bits, with exact scores."""
import numpy as np
import pytest

from tests.exact_scores import Exact, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wide", [False, True])          # (the cache holds values that fp16 does not: the other form)
@pytest.mark.parametrize("top", [-46, -4, -3, 0, 3, 14, 40])
@pytest.mark.parametrize("below", [10, 21, 22, 26])
def test_keys_far_below_the_largest(top, below, wide):
    """Every eighth key has a score of `top` (to the base 2) and a value of zero, the others are 2^-below of its probability: the result is theirs."""
    rng = np.random.default_rng(1)
    lens = [200, 64, 1, 100, 400]

    def message(i, n):
        large = np.arange(n) % 8 == 3 if n > 1 else np.ones(n, bool)
        return np.where(large, top, top - below), np.where(large[:, None], 0, 1 + rng.integers(0, 3, size=(n, 128)) / 2)
    layer = Exact([message(i, n) for i, n in enumerate(lens)] + ([(np.zeros(3), np.full((3, 128), 2.0 ** 20))] if wide else []))
    lists = [[0, 1, 2, 3, 4], [4, 0], [3, 1, 0, 2], [0, 4, 1]]
    c = layer.cache
    for rows, sharing, gather, window, static in [(1, 1, 0, 0, False), (1, 2, 0, 0, False), (1, 0, 0, 0, True), (2, 0, 1, 0, False), (5, 0, 1, 0, True), (40, 0, 1, 0, False),
                                                  (40, 0, 1, 1 << 20, False), (90, 0, 1, 0, True), (40, 0, 2, 0, False), (90, 0, 2, 0, False)]:
        c.set_decode_sharing(sharing)
        c.set_key_gather(gather)
        calls = [(m, rows) for m in lists]
        q = layer.query(4 * rows)
        close(layer.attend(calls, q, window, static), layer.want(calls, q), f"{rows} rows, sharing {sharing}, gather {gather}, window {window}, static {static}")
    c.close()
