"""Attention over PC_MX4 caches whose values are the largest and the smallest that they hold, with exact scores."""
import numpy as np
import pytest

from tests.exact_scores import Exact, close

pytestmark = pytest.mark.gpu

WAYS = [(1, 1, 0), (1, 2, 0), (2, 0, 1), (40, 0, 1), (90, 0, 1), (40, 0, 2), (90, 0, 2)]           # rows, sharing, gather


def every_way(layer, lists):
    for rows, sharing, gather in WAYS:
        layer.cache.set_decode_sharing(sharing)
        layer.cache.set_key_gather(gather)
        calls = [(m, rows) for m in lists]
        q = layer.query(len(lists) * rows)
        close(layer.attend(calls, q), layer.want(calls, q), f"{rows} rows, sharing {sharing}, gather {gather}")


@pytest.mark.parametrize("score", [20, 60, 63])
def test_largest_values_behind_smaller_scores(score):
    """Values of 6 x 2^60 whose scores are up to 2^63 times those in front of them, where a row's reference need not have moved yet: a sum of them
    without it would not fit 32 bits, and the result does."""
    layer = Exact([(np.zeros(64), np.full((64, 128), 1.5 * 2.0 ** 62)), (np.full(200, score), np.full((200, 128), 1.5 * 2.0 ** 62)),
                   (np.full(33, score - 2), np.full((33, 128), -2.0 ** 62))])
    every_way(layer, [[0, 1], [1], [1, 0, 2], [0, 2, 1]])
    layer.cache.close()


@pytest.mark.parametrize("score", [-20, -60, -62])
def test_smallest_values_at_small_scores(score):
    """Values about 2^-58 at scores that are themselves far below zero."""
    rng = np.random.default_rng(2)
    layer = Exact([(np.full(64, score), (1 + rng.integers(0, 3, size=(64, 128)) / 2) * 2.0 ** -58),
                   (np.full(200, score - 3), (2 + rng.integers(0, 3, size=(200, 128))) * 2.0 ** -60), (np.full(33, score - 8), np.full((33, 128), 2.0 ** -50))])
    every_way(layer, [[0, 1], [1], [1, 0, 2], [0, 2, 1]])
    layer.cache.close()


def test_values_about_the_border_of_the_copy():
    """Groups of eight that hold one value above the border, in every place, of messages that do not begin with a group: the call is right whichever way it goes."""
    rng = np.random.default_rng(5)
    messages = []
    for i, n in enumerate((13, 40, 7, 64, 100)):
        v = (1 + rng.integers(0, 3, size=(n, 128)) / 2) * 2.0 ** 24
        v[i::9] *= 4
        v[:, 32 * (i % 4):32 * (i % 4) + 32] /= 2.0 ** 10
        messages.append((rng.choice([0, -1, -2, 40], size=n), v))
    layer = Exact(messages)
    every_way(layer, [[0, 1, 2, 3, 4], [2, 0, 4], [3], [4, 2, 1]])
    layer.cache.close()
