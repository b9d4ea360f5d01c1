"""Long prefills over a copy of a PC_MX4 cache, in splits: values that 16-bit parts do not hold, and queries of no number."""
import numpy as np
import pytest

from tests.project_cases import Layer4, same

pytestmark = pytest.mark.gpu

LENS = [1100, 33, 900, 223]
SEL = [(0, 0), (2, 1200), (1, 2100), (3, 2200)]


def split(layer, calls, q):
    """The calls over a copy and in splits (class 8: a copy, class 4: a merge)."""
    layer.cache.profile_enable(True)
    out, lse = layer.attend(calls, q)
    of = list(layer.cache.profile_read().values())
    layer.cache.profile_enable(False)
    assert of[8][1] >= 1 and of[4][1] >= 1
    return out, lse


WAYS = [(2, 0, 200), (2, 3, 40), (0, 0, 1030)]           # (key gather, tiles a split as the caller says, rows): splits by every rule


@pytest.mark.parametrize("power", [20, 50, -12, -30])
def test_values_outside_fp16_over_a_copy_in_splits(power):
    """Parts of splits hold values that fp16 does not."""
    def spoil(i, k, v):
        v *= np.float32(2.0) ** power
    layer = Layer4(LENS, 16, 2, spoil=spoil)
    unit = 2.0 ** power
    for gather, tiles, rows in WAYS:
        layer.cache.set_key_gather(gather)
        layer.cache.set_tuning(0, tiles)
        calls = [(SEL, -1, 2500, rows)]
        q = layer.normal(rows, 16, 128)
        out, lse = split(layer, calls, q)
        want, want_lse = layer.want(calls, q)
        same(out.double() / unit, lse, want / unit, want_lse, f"values by 2^{power}, {rows} rows")
    layer.cache.close()


@pytest.mark.parametrize("what", ["NaN", "infinities at position 0", "both"])
def test_queries_that_are_no_numbers_over_a_copy_in_splits(what):
    """A row's head whose query holds a NaN or an infinity is NaN, its log-sum-exp too, and no other is touched: NaN of either sign, infinities where a
    turn's sine is zero and elsewhere, in first, middle and last rows and dims."""
    layer = Layer4(LENS, 16, 2)
    for gather, tiles, rows in WAYS:
        layer.cache.set_key_gather(gather)
        layer.cache.set_tuning(0, tiles)
        calls = [(SEL, -1, 0, rows)]
        q = layer.normal(rows, 16, 128)
        spoilt, bad = q.copy(), np.zeros((rows, 16), bool)
        places = {"NaN": [(0, 9, 127, np.nan), (31, 0, 64, -np.nan), (rows - 1, 15, 0, np.nan)], "infinities at position 0": [(0, 3, 5, np.inf), (0, 15, 127, -np.inf)],
                  "both": [(0, 3, 5, np.inf), (2, 9, 1, np.nan), (rows - 2, 15, 63, -np.inf)]}[what]
        for r, h, d, x in places:
            spoilt[r, h, d], bad[r, h] = x, True
        out, lse = split(layer, calls, spoilt)
        want, want_lse = layer.want(calls, q)
        some, rest = layer.torch.from_numpy(bad), layer.torch.from_numpy(~bad)
        assert out[some].isnan().all() and lse[some].isnan().all(), f"{rows} rows"
        same(out[rest], lse[rest], want[~bad], want_lse[~bad], f"{rows} rows")
    layer.cache.close()
