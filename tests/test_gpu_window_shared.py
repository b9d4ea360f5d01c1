"""pc_attend_window for single tokens of many calls over the same messages, which read every tile once (a workgroup multiplies it with
the queries of all calls that see it), against the fp64 oracle.  Whether calls go that way by themselves is a matter of cost; here they are
told to (pc_set_decode_sharing)."""
import numpy as np
import pytest

from tests.window_cases import Layer, compare, say

pytestmark = pytest.mark.gpu

LENS = [200, 31, 64, 333, 1, 150, 290, 97, 400, 128, 77, 260]


def agents(rng, n, n_msgs, n_lens, own0, some=0.8):
    """n calls of one row: most of the messages, in orders and at positions of their own; every third has an own message."""
    calls = []
    for i in range(n):
        order = [int(m) for m in rng.permutation(n_msgs) if rng.random() < some] if i % 2 else list(range(n_msgs))
        at, sel = int(rng.integers(0, 50)), []
        for m in order:
            sel.append((m, at))
            at += n_lens[m] + int(rng.integers(0, 3))
        calls.append((sel, own0 + i // 3 if i % 3 == 0 else -1, at, 1) if i % 3 == 0 else (sel, -1, at, 1))
    return calls


def run(layer, calls, window, n_sink, static=False):
    q = layer.normal(layer.rows(calls), layer.h_q, layer.D)
    out, lse = layer.attend(calls, window, n_sink, q, static)
    compare(layer.dtype, out, lse, *layer.want(calls, window, n_sink, q), f"w {window} s {n_sink} calls {len(calls)}")


# heads a KV head: 8 (two calls a group of columns), 1, 3 (a column to spare), 5, 16
@pytest.mark.parametrize("h_q,h_kv,n_calls", [(16, 2, 32), (16, 2, 7), (2, 2, 48), (3, 1, 23), (5, 1, 40), (16, 1, 20), (4, 1, 70)])
def test_calls_that_share_their_messages(h_q, h_kv, n_calls):
    rng = np.random.default_rng(n_calls)
    own = [int(x) for x in rng.integers(1, 40, size=(n_calls + 2) // 3)]
    layer = Layer("bf16", LENS + own, h_q, h_kv, 128)
    layer.cache.set_decode_sharing(2)
    calls = agents(rng, n_calls, len(LENS), LENS, len(LENS))
    for window, n_sink in [(1 << 30, 0), (900, 5), (700, 64), (2031, 300)]:
        run(layer, calls, window, n_sink)
    run(layer, calls, 1500, 33, static=True)
    layer.cache.close()


def test_long_and_short_messages_and_calls_that_see_little():
    """Messages longer than a workgroup's share and of one token; calls that see only the end, only the sinks, or nothing at all;
    prefill calls in between; the same message twice (those go their own way)."""
    rng = np.random.default_rng(5)
    lens = [3000, 1, 2500, 1, 33, 1900] + [20] * 4
    layer = Layer("bf16", lens, 16, 2, 128)
    layer.cache.set_decode_sharing(2)
    base = [(0, 0), (1, 3000), (2, 3001), (3, 5501), (4, 5502), (5, 5535)]
    calls = [(base, 6 + i % 4, 7435 + i, 1) for i in range(20)]
    calls[3:3] = [([(5, 0)], -1, 1900, 1), ([(0, 0)], -1, 0, 1, [10 ** 6]), (base[:2], -1, 0, 40, list(range(2900, 2940))), ([], 7, 0, 1), (base[::-1], -1, 9000, 1)]
    for window, n_sink in [(1 << 30, 0), (4000, 100), (2000, 3500), (1, 1)]:
        run(layer, calls, window, n_sink)
    twice = [(base + [(0, 9000)], -1, 12000 + i, 1) for i in range(24)]
    for window, n_sink in [(1 << 30, 0), (10000, 7)]:
        run(layer, twice, window, n_sink)
    layer.cache.close()


def test_what_is_not_finite_stays_with_the_calls_that_see_it():
    """Values and keys that some calls do not list, or do not see: nothing of them reaches their rows, though the tiles are shared."""
    def spoil(ks, vs):
        for i, m in enumerate((1, 4, 7)):
            vs[m][5::9, :, i::5] = [np.inf, np.nan, -np.inf][i]
            ks[m][3::11, 0, 5] = [np.nan, np.inf, np.nan][i]
    layer = Layer("bf16", [300] * 9 + [40], 16, 2, 128, spoil=spoil)
    layer.cache.set_decode_sharing(2)
    whole = [(m, 300 * m) for m in range(9)]
    clean = [e for e in whole if e[0] not in (1, 4, 7)]
    calls = [(whole if i % 3 == 2 else clean, 9 if i % 2 else -1, 2700, 1) for i in range(33)]
    # (window 500: rows at 2700 see messages 8 and a part of 7; window 290: message 8 alone)
    q = layer.normal(33, 16, 128)
    for window, n_sink, untouched in [(1 << 30, 0, lambda i: i % 3 != 2), (590, 0, lambda i: i % 3 != 2), (290, 0, lambda i: True), (290, 299, lambda i: True)]:
        out, lse = layer.attend(calls, window, n_sink, q)
        rows = [i for i in range(33) if untouched(i)]
        want, want_lse = layer.want([calls[i] for i in rows], window, n_sink, q[rows])
        compare("bf16", out[rows], lse[rows], want, want_lse, f"w {window} s {n_sink}")
        touched = [i for i in range(33) if not untouched(i)]
        if touched:
            assert not np.isfinite(out[touched].float().cpu().numpy()).all()
    layer.cache.close()


def test_each_way_gives_the_same():
    """A batch that shares its messages, and each of its calls alone."""
    rng = np.random.default_rng(9)
    layer = Layer("bf16", LENS, 16, 2, 128)
    layer.cache.set_decode_sharing(2)
    calls = [c for c in agents(rng, 24, len(LENS), LENS, 0) if c[1] < 0]
    q = layer.normal(len(calls), 16, 128)
    for window, n_sink in [(1 << 30, 0), (800, 10)]:
        layer.cache.set_decode_sharing(2)
        out, lse = layer.attend(calls, window, n_sink, q)
        again, _ = layer.attend(calls, window, n_sink, q)
        layer.cache.set_decode_sharing(1)
        own, own_lse = layer.attend(calls, window, n_sink, q)
        layer.cache.set_decode_sharing(0)
        assert (out.float() - own.float()).abs().max().item() <= 4e-2 and (lse - own_lse).abs().max().item() <= 2 * 2.0 ** -8
        assert bool((out == again).all())                # (no sum depends on an order that is not fixed)
        for i, c in enumerate(calls):
            o, l = layer.attend([c], window, n_sink, q[i:i + 1])
            # Both round the scores' operands alike.  The probabilities are rounded relative to a running maximum, which differs, and
            # the denominator sums the rounded ones: each is off by at most 2^-8 of itself, so either sum is, and the two
            # logarithms by at most 2 x 2^-8 of each other.
            far = (o.float() - out[i:i + 1].float()).abs().max().item()
            assert far <= 4e-2 and (l - lse[i:i + 1]).abs().max().item() <= 2 * 2.0 ** -8, (i, far)
    say("  the same")
    layer.cache.close()
