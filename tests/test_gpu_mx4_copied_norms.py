"""Long prefills over a copy of a PC_MX4 cache whose keys and queries are small or large for fp16, against 64 bits with exact scores."""
import numpy as np
import pytest

from tests.exact_scores import LN2, Exact, close

pytestmark = pytest.mark.gpu

FREE = list(range(32, 64)) + list(range(96, 128))        # dims that do not turn


def keys(rng, n, size):
    k = np.zeros((n, 128))
    k[:, FREE] = size * rng.choice([1, 1.5, 2, 3], size=(n, len(FREE)))
    return k


@pytest.mark.parametrize("size", [256, 16, 1])
def test_tiny_queries(size):
    """Queries below fp16's smallest number times keys that all have the same score: 64 products of one sign, so that what a query's value loses counts 64
    times.  A query's value is off by 2^-25 in the copy's walk at most: a score by 2^-25 x 2^10 x sqrt(128) where the keys' norm is 2^10 at most."""
    k = np.zeros((300, 128))
    k[:, FREE] = 3 * size
    layer = Exact([(k, np.ones((300, 128)))])
    tiny = 251 / 256 * 2.0 ** -25                        # (a bf16 number that fp16 rounds to zero)
    for gather in (1, 2):
        layer.cache.set_key_gather(gather)
        q = np.zeros((40, layer.h_q, 128))
        q[..., FREE] = tiny
        out, lse = layer.attend([([0], 40)], q)
        _, want_lse = layer.want([([0], 40)], q)
        score = 64 * 3 * size * tiny
        # in place: 2^-8 of the score; over the copy what is said above; 3e-6: of a logarithm in 32 bits
        bar = LN2 * (2.0 ** -8 * score if gather == 1 else min(score, 2.0 ** -25 * 2 ** 10 * 128 ** 0.5)) + 3e-6
        assert (out == 1).all() and np.abs(lse - want_lse).max() <= bar, (gather, np.abs(lse - want_lse).max(), bar)
    layer.cache.close()


@pytest.mark.parametrize("size", [64, 128, 600, 2.0 ** 12, 2.0 ** 30, 2.0 ** 55])
def test_large_keys(size):
    """A few keys of a large norm among many of an ordinary one: they take all of a row, or have nothing of it, and every row is as it should be."""
    rng = np.random.default_rng(3)
    size = 2.0 ** np.floor(np.log2(size))
    k = keys(rng, 300, 0.125)
    k[:, FREE] *= rng.choice([-1, 1], size=(300, len(FREE)))
    k[[17, 130, 131, 299]] = keys(rng, 4, size)
    v = rng.integers(1, 5, size=(300, 128)) / 2
    layer = Exact([(k, v)])
    q = np.zeros((80, layer.h_q, 128))
    for r in range(80):
        q[r, :, rng.choice(FREE, size=8, replace=False)] = rng.choice([1, 2], size=(8, layer.h_q))
    q[1::2] *= -1
    for gather in (1, 2):
        layer.cache.set_key_gather(gather)
        # (probabilities are no powers of two here: rounded to bf16 in the copy's walk, numerator and, but for the last tile, not the denominator)
        close(layer.attend([([0], 80)], q), layer.want([([0], 80)], q), f"keys of {size}, gather {gather}", bar=2.0 ** -7 + 2.0 ** -9, lse_bar=2.0 ** -8)
    layer.cache.close()


@pytest.mark.parametrize("size", [2.0 ** 6, 2.0 ** 8, 2.0 ** 12, 2.0 ** 40, 2.0 ** 100])
def test_large_queries(size):
    """Some rows of a large norm: one key, or those that are alike, take all of it."""
    rng = np.random.default_rng(4)
    k = keys(rng, 300, 0.25)
    k[:, FREE] *= rng.choice([-1, 1], size=(300, len(FREE)))
    v = rng.integers(1, 5, size=(300, 128)) / 2
    layer = Exact([(k, v)])
    q = np.zeros((80, layer.h_q, 128))
    for r in range(80):
        q[r, :, rng.choice(FREE, size=8, replace=False)] = rng.choice([1, 2, -1], size=(8, layer.h_q))
    q[::7] *= size
    for gather in (1, 2):
        layer.cache.set_key_gather(gather)
        close(layer.attend([([0], 80)], q), layer.want([([0], 80)], q), f"queries of {size}, gather {gather}", bar=2.0 ** -7 + 2.0 ** -9, lse_bar=2.0 ** -8)
    layer.cache.close()
